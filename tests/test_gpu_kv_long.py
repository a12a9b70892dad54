"""atp_kv_attend where contexts are long enough for what short ones never reach
(GPU, through the C ABI, against the 64-bit oracle): chunks above the shortest
length and waves of several steps, two rounds of chunks, lengthened chunks;
chunks and parts of tiles in which a row sees nothing; the precision that the
few-row kernel claims; valid sequences beside refused ones."""
import numpy as np
import pytest
import torch

from oracle import kvstep
from paper_2511_11617_amd import atp
from tests.test_gpu_kv_ops import E, GQA, TORCH, Setup

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def few_check(s, out, lse, **m):
    """As Setup.check, with the few-row kernel's own error: its weights enter
    the second product as two 16-bit parts, off by u^2 of themselves; in fp16
    the largest is at least 2^7 and the second part's least step 2^-24, so a
    weight is off by 2^-25 / 2^7 = 2^-32 of the largest besides."""
    K, V, seen = s.contexts()
    scale, cap, slopes = m.get("scale", s.hd ** -0.5), m.get("softcap", 0.0), m.get("slopes")
    want, want_lse, weight, reach = kvstep.attend(s.q.double().cpu().numpy(), K, V, s.starts.tolist(), s.cached, s.q_heads, s.kv_heads,
                                                  s.group, scale, cap, m.get("window", 0), slopes, seen)
    u, n = torch.finfo(TORCH[s.dtype]).eps / 2, max(c + f for c, f in zip(s.cached, s.fresh))
    ds = (s.hd + 8) * E * reach + 16 * E * reach + (cap * 2.0 ** -21 if cap else 0)
    rel = u * u + 2 * ds + (n + 64) * E
    tol = u * np.abs(want) + 1.1 * weight * rel[..., None]
    if s.dtype == "fp16":
        tol += 2.0 ** -25 + n * 2.0 ** -32 * max(np.abs(v).max() for v in V)
    got, rows = out.double().cpu().numpy(), int(s.starts[-1])
    off = np.abs(got - want)[:rows] / tol[:rows]
    assert off.max() <= 1, float(off.max())
    l = np.abs(lse.double().cpu().numpy() - want_lse)[:rows]
    assert np.all(l <= (ds + (n + 64) * E + 4 * E * np.abs(want_lse))[:rows])


def chunking(s):
    """Tokens of the few-row kernel's chunks, its rounds, and whether chunks were lengthened for sequences' short ends."""
    per_head, runs = max(s.fresh) * min(s.group, s.n_q), s.n_kv
    groups = 256 if s.hd > 128 or (s.hd > 64 and per_head > 16) else 512 if s.hd > 64 else 768
    spans = [c + f if f else 0 for c, f in zip(s.cached, s.fresh)]
    rounds = 2 if len(spans) * runs > groups else 1
    each = -(-sum(spans) * runs // (rounds * groups))
    chunk = max(256, -(-each // 64) * 64)
    n = sum(-(-x // chunk) for x in spans) * runs
    longer = len(spans) <= 256 and chunk > 256 and n > rounds * groups * 9 // 8
    return -(-(each + each // 3) // 64) * 64 if longer else chunk, rounds, longer


ONE_RUN = dict(q_heads=(8, 14), kv_heads=(1, 2), group=8)
LONG = {  # what it is to reach: (steps of its busiest wave, rounds, lengthened)
    "steps": (dict(cached=[7000 - 31 * i for i in range(20)], fresh=[1] * 20, **GQA), (5, 1, False)),
    "steps_odd": (dict(cached=[4900 - 17 * i for i in range(20)], fresh=[1] * 20, layout="token", dtype="fp16", **GQA), (3, 1, False)),
    "steps_e4m3": (dict(cached=[9500 - 41 * i for i in range(20)], fresh=[1] * 20, cache="e4m3", **GQA), (3, 1, False)),
    "steps_64": (dict(cached=[9100 - 53 * i for i in range(20)], fresh=[1] * 20, hd=64, layout="token", **GQA), (4, 1, False)),
    "steps_drafts": (dict(cached=[7600 - 31 * i for i in range(8)], fresh=[4, 3, 4, 1, 0, 4, 2, 4], **GQA), (4, 1, False)),
    "steps_256": (dict(cached=[7300 - 31 * i for i in range(8)], fresh=[2, 1] * 4, hd=256, **GQA), (4, 1, False)),
    "steps_blocks_of_5": (dict(cached=[7600 - 31 * i for i in range(8)], fresh=[3] * 8, bt=5, hd=80, **GQA), (4, 1, False)),
    "two_rounds": (dict(cached=[(97 * i) % 1201 for i in range(130)], fresh=[4 - i % 3 for i in range(130)], **GQA), (4, 2, True)),
    "two_rounds_64": (dict(cached=[(97 * i) % 1201 for i in range(400)], fresh=[1] * 400, hd=64, dtype="fp16", layout="token", **GQA), (3, 2, False)),
    "lengthened": (dict(cached=[320 * (1 + i % 4) + 10 for i in range(100)], fresh=[5] * 100, **ONE_RUN), (4, 1, True)),
}


@pytest.mark.parametrize("name", LONG)
def test_chunks_of_several_steps(name):
    kw, (steps, rounds, longer) = LONG[name]
    s = Setup(**kw, seed=31)
    chunk, got_rounds, got_longer = chunking(s)
    step = 64 if s.e4m3 and s.hd <= 128 else 32
    assert (-(-chunk // (4 * step)), got_rounds, got_longer) == (steps, rounds, longer), (chunk, got_rounds, got_longer)
    out, lse = s.attend()
    few_check(s, out, lse)


@pytest.mark.parametrize("mask", [dict(softcap=5.0), dict(window=1500)])
def test_chunks_of_several_steps_with_a_mask(mask):
    s = Setup(**LONG["steps_drafts"][0], seed=32)
    out, lse = s.attend(**mask)
    few_check(s, out, lse, **mask)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape,scale", [(dict(cached=[300, 5, 0], fresh=[1, 1, 1]), 128 ** -0.5), (dict(cached=[900], fresh=[4]), 128 ** -0.5),
                                         (dict(cached=[700], fresh=[1], hd=256), 1 / 16), (dict(cached=[40] * 9, fresh=[1] * 9), 2 ** -9)])
def test_few_rows_lose_nothing_of_the_weights(shape, scale, dtype, cache):
    """Weights of one 16-bit part would be off by 1.6 times this in bf16 (300
    tokens), and by 15 and 8 times it in bf16 and fp16 where scores and contexts
    are small."""
    s = Setup(**shape, **GQA, dtype=dtype, cache=cache, seed=33)
    out, lse = s.attend(scale=scale)
    few_check(s, out, lse, scale=scale)


GAPS = {"decode": dict(cached=[6000, 900, 2000], fresh=[1, 1, 1]), "drafts": dict(cached=[6000, 900, 2000], fresh=[4, 2, 1]),
        "prompt": dict(cached=[6000, 900, 2000], fresh=[40, 9, 33])}


@pytest.mark.parametrize("dtype,cache", [("bf16", "same"), ("fp16", "same"), ("bf16", "e4m3")])
@pytest.mark.parametrize("shape", GAPS)
def test_gaps_wider_than_a_chunk_or_part(shape, dtype, cache):
    """Absent blocks and bad ids over whole chunks, with NaN wherever nothing is
    seen: at the begin, in the middle, up to the new tokens, and over a whole
    sequence."""
    s = Setup(**GAPS[shape], **GQA, dtype=dtype, cache=cache, seed=34)
    t = s.table.copy()
    t[0, :40] = -1                                   # tokens 0 to 639
    t[0, 100:260] = -1                               # 1600 to 4159
    t[0, 150:200] = [s.pool, -5, 2 ** 31 - 1, -2 ** 31, s.pool + 1] * 10
    t[1, :] = -1                                     # all of it
    t[2, 20:(s.cached[2] + s.fresh[2] + 15) // 16] = -1  # 320 to its end
    s.d_table.copy_(torch.from_numpy(t))
    live = torch.zeros(s.pool, dtype=torch.bool)
    live[torch.from_numpy(t[(t >= 0) & (t < s.pool)]).long()] = True
    a = s.arena.view(torch.uint8) if s.e4m3 else s.arena
    clean = s.arena.clone()
    a[:, :, ~live.cuda()] = 0x7F if s.e4m3 else float("nan")
    out, lse = s.attend()
    s.arena.copy_(clean)
    s.check(out, lse, table=t)
    r = slice(s.starts[1], s.starts[2])
    assert bool((out[r] == 0).all()) and bool(torch.isneginf(lse[r]).all())
    assert s.status.tolist()[0] == atp.EINVAL


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_parts_that_a_window_leaves_empty_for_some_rows(dtype):
    """A prompt's tile that is cut: its first and last rows see different parts."""
    s = Setup(cached=[3000], fresh=[600], q_heads=(0, 2), kv_heads=(0, 2), group=1, dtype=dtype, seed=35)
    for window in (1, 100, 1000):
        out, lse = s.attend(window=window)
        s.check(out, lse, window=window)


@pytest.mark.parametrize("what", ["cached", "fresh", "ctx", "rows"])
@pytest.mark.parametrize("fresh", [[1, 2, 1], [3, 40, 20], [30, 40, 20]])
def test_sequences_beside_one_that_breaks_a_bound_are_right(what, fresh):
    s = Setup(cached=[340, 850, 860], fresh=fresh, **GQA, pad=1, bounds=(max(fresh), 860 + max(fresh)))
    rows, left = s.rows, [1]
    if what == "cached":
        s.d_cached[1] = -1
    elif what == "fresh":
        s.step.d.max_fresh = fresh[1] - 1
    elif what == "ctx":
        s.step.d.max_ctx, left = 860 + fresh[2] - 1, [2] + [1] * (850 + fresh[1] >= 860 + fresh[2])
    else:
        s.step.d.max_tokens, left = rows - 2, [2]
    out, lse = s.attend()
    good = [r for q in range(3) if q not in left for r in range(s.starts[q], s.starts[q + 1])]
    s.check(out, lse, rows=np.array(good))
    bad = [r for q in left for r in range(s.starts[q], s.starts[q + 1])]
    assert bool((out[bad] == 7).all()) and bool((lse[bad] == 7).all()) and s.status.tolist()[0] == atp.EINVAL

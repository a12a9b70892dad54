"""KV cache operators on the GPU (through the C ABI) against the 64-bit oracle.

Tolerances follow from the arithmetic: u = eps / 2 is one rounding to the
output's type, e = 2^-24 one to 32 bits.  Attention: a score is a sum of dim
products and a few more operations, off by at most
  ds = (dim + 8) e reach + 16 e |score| (+ cap * 2^-21 under a tanh),
so a weight is off by 2 ds relative, and by u where it is rounded to the
type; sums over n tokens add n e; the output is rounded once more.
"""
import math

import numpy as np
import pytest
import torch

from oracle import kvstep
from paper_2511_11617_amd import atp

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16}
CODE = {"bf16": atp.BF16, "fp16": atp.FP16}


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def dev(x, dtype):
    return torch.tensor(x, dtype=dtype, device="cuda")


def stream():
    return torch.cuda.current_stream().cuda_stream


class Setup:
    """A cache of one rank and one step's requests, with host copies."""

    def __init__(self, cached, fresh, q_heads=(0, 8), kv_heads=(0, 1), group=8, hd=128, bt=16, layout="head", dtype="bf16",
                 cache="same", layers=1, pad=0, spare=1, seed=0, pool_extra=5, bounds=None, grow=0):
        self.rng = np.random.default_rng(seed)
        self.cached, self.fresh, self.q_heads, self.kv_heads, self.group = list(cached), list(fresh), q_heads, kv_heads, group
        self.hd, self.bt, self.layout, self.dtype, self.layers = hd, bt, layout, dtype, layers
        self.n_q, self.n_kv = q_heads[1] - q_heads[0], kv_heads[1] - kv_heads[0]
        n = len(cached)
        self.rows = sum(fresh) + pad
        need = [-(-(c + f) // bt) for c, f in zip(cached, fresh)]
        self.max_blocks = max(need + [1]) + spare
        self.pool = sum(need) + pool_extra + grow
        ids = self.rng.permutation(self.pool)
        self.table = np.full((n, self.max_blocks), -1, np.int32)
        at = 0
        for s, k in enumerate(need):
            self.table[s, :k] = ids[at:at + k]
            at += k
        self.starts = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
        self.e4m3 = cache == "e4m3"
        g = torch.Generator().manual_seed(seed)
        shape = (layers, 2, self.pool, self.n_kv, bt, hd) if layout == "head" else (layers, 2, self.pool, bt, self.n_kv, hd)
        x = torch.randn(shape, generator=g)
        self.arena = ((x * 32).to(torch.float8_e4m3fn) if self.e4m3 else x.to(TORCH[dtype])).cuda()
        self.scales = (torch.rand(layers, 2, self.n_kv, generator=g) + 0.5).div(32).cuda() if self.e4m3 else None
        self.d_table, self.d_starts = dev(self.table, torch.int32), dev(self.starts, torch.int32)
        self.d_cached, self.d_fresh = dev(cached, torch.int32), dev(fresh, torch.int32)
        self.status = torch.zeros(4, dtype=torch.int32, device="cuda")
        slots, pos = np.full(self.rows, -1, np.int64), np.zeros(self.rows, np.int32)
        for s in range(n):
            for i in range(fresh[s]):
                p = cached[s] + i
                slots[self.starts[s] + i], pos[self.starts[s] + i] = int(self.table[s, p // bt]) * bt + p % bt, p
        self.slots, self.positions = slots, pos
        self.d_slots, self.d_pos = dev(slots, torch.int64), dev(pos, torch.int32)
        mf, mc = bounds or (max(list(fresh) + [0]), max([c + f for c, f in zip(cached, fresh)] + [0]))
        self.step = atp.KVStep(self.d_table.data_ptr(), n, self.max_blocks, self.d_cached.data_ptr(), self.d_fresh.data_ptr(),
                               self.d_starts.data_ptr(), self.d_slots.data_ptr(), self.d_pos.data_ptr(), self.rows, mf, mc,
                               self.status.data_ptr())
        self.cache = atp.KVCache(self.arena.data_ptr(), self.arena.numel() * self.arena.element_size(), layers, bt, hd, self.pool,
                                 q_heads, kv_heads, group, CODE[dtype], atp.E4M3 if self.e4m3 else None,
                                 atp.KV_HEAD_MAJOR if layout == "head" else atp.KV_TOKEN_MAJOR,
                                 self.scales.data_ptr() if self.e4m3 else 0)
        self.q = torch.randn(self.rows, self.n_q, hd, generator=g).to(TORCH[dtype]).cuda()

    def heads_first(self, layer=0):
        """float64 [2, pool, KV heads, block_tokens, dim]"""
        a = self.arena[layer].float().double().cpu().numpy()
        if self.layout == "token":
            a = a.transpose(0, 1, 3, 2, 4)
        if self.e4m3:
            a = a * self.scales[layer].double().cpu().numpy()[:, None, :, None, None]
        return a

    def contexts(self, layer=0, table=None):
        """Per sequence: K, V [context, KV heads, dim] and which tokens are there."""
        a, table = self.heads_first(layer), self.table if table is None else table
        K, V, seen = [], [], []
        for s in range(len(self.cached)):
            t = np.arange(self.cached[s] + self.fresh[s])
            p = table[s, t // self.bt]
            ok = (p >= 0) & (p < self.pool)
            p = np.where(ok, p, 0)
            K.append(a[0][p, :, t % self.bt])
            V.append(a[1][p, :, t % self.bt])
            seen.append(ok)
        return K, V, seen

    def attend(self, layer=0, scale=None, softcap=0.0, window=0, slopes=None, want_lse=True, q=None, out=None):
        q = self.q if q is None else q
        out = torch.full((self.rows, self.n_q, self.hd), 7.0, dtype=TORCH[self.dtype], device="cuda") if out is None else out
        lse = torch.full((self.rows, self.n_q), 7.0, device="cuda") if want_lse else None
        d_slopes = dev(slopes, torch.float32) if slopes is not None else None
        mask = atp.Mask(self.hd ** -0.5 if scale is None else scale, softcap, window, d_slopes.data_ptr() if slopes is not None else 0)
        need = atp.kv_attend_workspace(self.cache, self.step)
        ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")  # every float in it a NaN
        atp.kv_attend(self.cache, self.step, layer, mask, q.data_ptr(), q.stride(0), out.data_ptr(), out.stride(0),
                      lse.data_ptr() if want_lse else 0, ws.data_ptr(), need, stream())
        torch.cuda.synchronize()
        assert bool((ws[need:] == 0xFF).all()), "written past the workspace"
        return out, lse

    def check(self, out, lse, layer=0, scale=None, softcap=0.0, window=0, slopes=None, table=None, rows=None):
        scale = self.hd ** -0.5 if scale is None else scale
        K, V, seen = self.contexts(layer, table)
        sl = None if slopes is None else np.float32(slopes).astype(np.float64)
        want, want_lse, weight, reach = kvstep.attend(self.q.double().cpu().numpy(), K, V, self.starts.tolist(), self.cached,
                                                      self.q_heads, self.kv_heads, self.group, scale, softcap, window, sl, seen)
        u = torch.finfo(TORCH[self.dtype]).eps / 2
        n = max(c + f for c, f in zip(self.cached, self.fresh))
        top = reach.copy()
        if slopes is not None:
            top += np.abs(sl)[None, :] * n
        ds = (self.hd + 8) * E * reach + 16 * E * top + (softcap * 2.0 ** -21 if softcap else 0)
        rel = u + 2 * ds + (n + 64) * E
        # fp16: weights below 2^-29 of the largest lose bits, 2^-40 of it at most, n of them
        tol = u * np.abs(want) + 1.1 * weight * rel[..., None] + n * 2.0 ** -39 + (2.0 ** -25 if self.dtype == "fp16" else 0)
        rows = np.arange(int(self.starts[-1])) if rows is None else rows
        got, pad = out.double().cpu().numpy(), slice(int(self.starts[-1]), None)
        off = np.abs(got - want)[rows]
        assert np.all(off <= tol[rows]), (float(np.nanmax(off)), float(np.nanmax(off / tol[rows])), int((~(off <= tol[rows])).sum()))
        assert np.all(got[pad] == 7.0)
        if lse is not None:
            l = lse.double().cpu().numpy()
            assert np.all(l[pad] == 7.0)
            empty = np.isneginf(want_lse)
            assert np.array_equal(np.isneginf(l[rows]), empty[rows])
            with np.errstate(invalid="ignore"):
                lo = np.where(empty, 0, np.abs(l - want_lse))
            ltol = ds + (n + 64) * E + 4 * E * np.where(empty, 0, np.abs(want_lse))
            assert np.all(lo[rows] <= ltol[rows]), float((lo[rows] / ltol[rows]).max())


# ---- atp_kv_attend ---------------------------------------------------------------
GQA = dict(q_heads=(10, 19), kv_heads=(1, 3), group=8)  # runs of 6 and 3 query heads

ATTEND = {
    "one_token": dict(cached=[0], fresh=[1]),
    "tiny": dict(cached=[127, 0, 15, 16, 31, 64, 100, 3], fresh=[1] * 8, q_heads=(0, 2), group=2, hd=64, dtype="fp16", pad=3),
    "runs": dict(cached=[500, 77, 0, 1000, 255, 256, 257], fresh=[1] * 7, **GQA),
    "runs_token": dict(cached=[500, 77, 0, 1000], fresh=[1] * 4, layout="token", **GQA),
    "no_group": dict(cached=[33, 95], fresh=[1, 1], q_heads=(2, 5), kv_heads=(2, 5), group=1),
    "many_heads_one_kv": dict(cached=[300, 20], fresh=[1, 1], q_heads=(0, 64), kv_heads=(0, 1), group=64),
    "odd_group": dict(cached=[130, 61], fresh=[1, 1], q_heads=(3, 30), kv_heads=(0, 5), group=7),
    "long": dict(cached=[20011], fresh=[1], q_heads=(4, 9), kv_heads=(0, 2), group=5),
    "long_ragged_e4m3": dict(cached=[9000, 1, 4097], fresh=[1, 1, 1], cache="e4m3", layout="token", **GQA),
    "e4m3": dict(cached=[70, 333], fresh=[1, 1], cache="e4m3", **GQA),
    "e4m3_fp16": dict(cached=[70, 333], fresh=[1, 2], cache="e4m3", dtype="fp16", **GQA),
    "drafts": dict(cached=[100, 0, 15, 49], fresh=[3, 2, 5, 0], pad=2, **GQA),
    "drafts_many": dict(cached=[100, 700], fresh=[7, 6], q_heads=(0, 16), kv_heads=(0, 2), group=8),
    "dim_8": dict(cached=[40], fresh=[2], hd=8, q_heads=(0, 3), group=3),
    "dim_72": dict(cached=[100, 5], fresh=[1, 2], hd=72, q_heads=(1, 6), kv_heads=(0, 2), group=4, bt=8),
    "dim_80": dict(cached=[100, 5, 1300], fresh=[1, 1, 1], hd=80, layout="token", q_heads=(1, 6), kv_heads=(0, 2), group=4),
    "dim_256": dict(cached=[100, 500], fresh=[1, 3], hd=256, q_heads=(0, 4), group=4),
    "dim_256_e4m3": dict(cached=[100, 500], fresh=[1, 30], hd=256, q_heads=(0, 4), group=4, cache="e4m3"),
    "blocks_of_1": dict(cached=[37], fresh=[2], bt=1),
    "blocks_of_5": dict(cached=[37, 101], fresh=[2, 1], bt=5, **GQA),
    "blocks_of_24": dict(cached=[37, 101], fresh=[40, 90], bt=24, **GQA),
    "blocks_of_256": dict(cached=[37, 300], fresh=[2, 1], bt=256, layout="token"),
    "prompt": dict(cached=[0], fresh=[200], **GQA),
    "prompt_fp16": dict(cached=[0, 3], fresh=[129, 64], dtype="fp16", q_heads=(0, 4), kv_heads=(0, 2), group=2, hd=64, pad=5),
    "prompt_behind": dict(cached=[333, 1000, 0], fresh=[65, 100, 33], layout="token", q_heads=(14, 27), kv_heads=(2, 6), group=5),
    "prompt_ragged": dict(cached=[0, 90, 500, 2, 0], fresh=[150, 1, 0, 17, 40], **GQA),
    "prompt_80": dict(cached=[50, 0], fresh=[70, 33], hd=80, q_heads=(1, 6), kv_heads=(0, 2), group=4, bt=8),
    "prompt_256": dict(cached=[50, 0], fresh=[70, 33], hd=256, q_heads=(0, 3), kv_heads=(0, 1), group=3),
    "prompt_e4m3": dict(cached=[100, 0], fresh=[60, 90], cache="e4m3", **GQA),
    "prompt_e4m3_fp16": dict(cached=[100, 0], fresh=[60, 90], cache="e4m3", dtype="fp16", hd=64, layout="token", **GQA),
    "chunk_behind_much": dict(cached=[6000], fresh=[40], q_heads=(0, 4), group=4),
    "two_layers": dict(cached=[40, 9], fresh=[1, 20], layers=3, **GQA),
    "mixed_batch": dict(cached=[0, 3000] + [20 * i for i in range(38)], fresh=[300, 1] + [1] * 30 + [0, 2] * 4, pad=7, **GQA),
    "prompt_behind_fp16_token": dict(cached=[2000, 31], fresh=[50, 70], dtype="fp16", layout="token", bt=32, **GQA),
    "prompt_of_one_head": dict(cached=[100], fresh=[300], q_heads=(2, 3), kv_heads=(1, 2), group=2),
    "many_sequences": dict(cached=[(37 * i) % 90 for i in range(600)], fresh=[1] * 600, q_heads=(0, 2), group=2, hd=64),
    "many_sequences_some_long": dict(cached=[(37 * i) % 90 + 1500 * (i % 97 == 5) for i in range(300)], fresh=[1 - (i % 11 == 3) for i in range(300)],
                                     q_heads=(1, 4), kv_heads=(0, 2), group=2, hd=64, layout="token"),
    "more_tiles_than_a_list": dict(cached=[i % 7 for i in range(4100)], fresh=[40] + [1] * 4099, q_heads=(0, 1), group=1, hd=64),
    "loose_bounds": dict(cached=[500, 77], fresh=[1, 2], bounds=(64, 5000), **GQA),
    "loose_bounds_one": dict(cached=[500, 77], fresh=[1, 1], bounds=(1, 40000), **GQA),
}


@pytest.mark.parametrize("name", ATTEND)
def test_attend(name):
    s = Setup(**ATTEND[name])
    layer = s.layers - 1
    out, lse = s.attend(layer)
    s.check(out, lse, layer)
    assert s.status.tolist() == [0, 0, 0, 0]


MASKS = {
    "softcap": dict(softcap=5.0), "softcap_small": dict(softcap=0.25, scale=3.0), "window_1": dict(window=1),
    "window_33": dict(window=33), "window_large": dict(window=100000), "window_largest": dict(window=2 ** 31 - 1), "slopes": dict(slopes=True),
    "all": dict(softcap=20.0, window=70, slopes=True, scale=0.3), "scale_0": dict(scale=0.0), "scale_negative": dict(scale=-0.2),
    "sharp": dict(scale=8.0),
}


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("shape", ["decode", "drafts", "prompt", "long", "behind"])
def test_attend_masks(shape, mask):
    kw = {"decode": dict(cached=[300, 40, 0], fresh=[1, 1, 1]), "drafts": dict(cached=[200, 31], fresh=[4, 2], dtype="fp16"),
          "prompt": dict(cached=[70, 0], fresh=[90, 140]), "behind": dict(cached=[1700, 40], fresh=[40, 9], dtype="fp16"), "long": dict(cached=[5000, 3100], fresh=[1, 1], layout="token")}[shape]
    s = Setup(**kw, **GQA, seed=3)
    m = dict(MASKS[mask])
    if m.get("slopes"):
        m["slopes"] = [2.0 ** (-1 - 0.5 * h) for h in range(s.n_q)]
    out, lse = s.attend(**m)
    s.check(out, lse, **m)


SHAPES = {"decode": dict(cached=[100, 61, 2000], fresh=[1, 1, 1]), "drafts": dict(cached=[100, 61], fresh=[3, 2]),
          "prompt": dict(cached=[100, 0], fresh=[80, 150])}


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("shape", SHAPES)
def test_attend_without_some_blocks(shape, cache):
    """Absent blocks (-1) inside the context are unseen, whatever block 0 or any other holds; a row that sees nothing is 0."""
    s = Setup(**SHAPES[shape], **GQA, cache=cache, seed=5, layout="token")
    t = s.table.copy()
    t[0, 1:3] = -1
    t[0, 5] = -1
    t[1, :(s.cached[1] + s.fresh[1] + 15) // 16] = -1  # nothing of sequence 1 is there
    s.d_table.copy_(torch.from_numpy(t))
    out, lse = s.attend()
    s.check(out, lse, table=t)
    r = slice(s.starts[1], s.starts[2])
    assert bool((out[r] == 0).all()) and bool(torch.isneginf(lse[r]).all()) and s.status.tolist()[0] == 0


@pytest.mark.parametrize("shape", SHAPES)
def test_attend_reports_bad_block_ids(shape):
    """An id outside the pool counts as absent and sets the status; the kernels never follow it."""
    s = Setup(**SHAPES[shape], **GQA, seed=6)
    t = s.table.copy()
    t[0, 1], t[0, 3], t[1, 0] = s.pool, 2 ** 31 - 1, -7
    s.d_table.copy_(torch.from_numpy(t))
    out, lse = s.attend()
    s.check(out, lse, table=t)
    assert s.status.tolist()[0] == atp.EINVAL


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("shape", list(SHAPES) + ["window"])
def test_attend_ignores_what_it_does_not_see(shape, cache):
    """NaN and infinity behind the context, in free blocks, before the window and in later tokens of the same step."""
    kw = SHAPES["prompt" if shape == "window" else shape]
    s = Setup(**kw, **GQA, cache=cache, seed=7)
    a = s.arena.view(torch.uint8) if s.e4m3 else s.arena
    nan = 0x7F if s.e4m3 else float("nan")
    live = torch.zeros(s.pool * s.bt, dtype=torch.bool)
    for q in range(len(s.cached)):
        for t in range(s.cached[q] + s.fresh[q]):
            live[int(s.table[q, t // 16]) * 16 + t % 16] = True
    dead = (~live).reshape(s.pool, 16).cuda()
    a.copy_(torch.where(dead[None, None, :, None, :, None], torch.full_like(a, nan), a))
    clean = s.arena.clone()
    window = 30 if shape == "window" else 0

    def spoil(seq, t, bad=nan):
        p, o = int(s.table[seq, t // 16]), t % 16
        a[0, :, p, :, o] = bad
        a[0, 1, p, :, o, ::3] = bad
        if not s.e4m3:
            a[0, 1, p, 0, o, 0], a[0, 1, p, 0, o, 1] = float("inf"), -float("inf")

    rows = []  # rows that see no spoilt token
    for q in range(len(s.cached)):
        last = s.cached[q] + s.fresh[q] - 1
        if shape == "window":
            spoil(q, 3)
            rows += [s.starts[q] + i for i in range(s.fresh[q]) if s.cached[q] + i - 3 >= 30 or s.cached[q] + i < 3]
        elif s.fresh[q] > 1:
            spoil(q, last)
            rows += list(range(s.starts[q], s.starts[q + 1] - 1))
        else:
            rows += [s.starts[q]]
    out, lse = s.attend(window=window)
    spoilt = torch.ones(s.rows, dtype=torch.bool)
    spoilt[rows] = False
    got = out.double().cpu()
    if shape != "decode":
        assert bool(torch.isnan(got[spoilt]).flatten(1).any(1).all()), "a row that sees a NaN shows it"
    s.arena.copy_(clean)
    s.check(out, lse, window=window, rows=np.array(rows))


def test_attend_seen_infinities_in_v():
    """A seen infinity in V reaches exactly the rows and dimensions that see it."""
    s = Setup(cached=[5], fresh=[40], q_heads=(0, 2), group=2, seed=9)
    p, o = int(s.table[0, 20 // 16]), 20 % 16
    s.arena[0, 1, p, 0, o, 3], s.arena[0, 1, p, 0, o, 4] = float("inf"), -float("inf")
    out, _ = s.attend()
    got = out.float().cpu()
    sees = torch.arange(40) + 5 >= 20
    assert bool((got[sees][:, :, 3] == math.inf).all()) and bool((got[sees][:, :, 4] == -math.inf).all())
    assert bool(torch.isfinite(got[~sees]).all())
    keep = [d for d in range(128) if d not in (3, 4)]
    assert bool(torch.isfinite(got[:, :, keep]).all())


def test_attend_strides_and_no_lse():
    s = Setup(cached=[90, 4], fresh=[1, 30], **GQA, seed=8)
    wide = torch.randn(s.rows, 3 * s.n_q * s.hd + 8, device="cuda").to(torch.bfloat16)
    q, out = wide[:, :s.n_q * s.hd], wide[:, s.n_q * s.hd:2 * s.n_q * s.hd]
    q.copy_(s.q.reshape(s.rows, -1))
    rest = wide[:, 2 * s.n_q * s.hd:].clone()
    s.attend(q=q, out=out, want_lse=False)
    s.check(out.reshape(s.rows, s.n_q, s.hd), None)
    assert torch.equal(wide[:, 2 * s.n_q * s.hd:], rest) and torch.equal(q, s.q.reshape(s.rows, -1))


@pytest.mark.parametrize("what", ["starts", "cached", "fresh", "ctx", "rows"])
def test_attend_leaves_sequences_that_break_a_bound(what):
    s = Setup(cached=[40, 50, 60], fresh=[1, 2, 1], **GQA, pad=1, bounds=(2, 61))
    if what == "starts":
        s.d_starts.copy_(torch.tensor([0, 1, 0, 1]))  # sequence 1 ends before it begins
        left = [3]
    elif what == "cached":
        s.d_cached[1] = -1
        left = [1, 2]
    elif what == "fresh":
        s.step.d.max_fresh, left = 1, [1, 2]
    elif what == "ctx":
        s.step.d.max_ctx, left = 60, [3]
    else:
        s.step.d.max_tokens, left = 3, [3]
    out, lse = s.attend()
    assert s.status.tolist()[0] == atp.EINVAL
    assert bool((out[left] == 7).all()) and bool((lse[left] == 7).all())
    s.status.zero_()


def test_attend_takes_offsets_past_32_bits():
    """The last blocks of an arena of more than 4 GiB."""
    hd, bt, n_kv, pool = 128, 64, 4, 20000  # 64 KiB a block and K|V plane of 1.3 GB
    layers = 2
    plane = pool * n_kv * bt * hd
    arena = torch.empty(layers * 2 * plane, dtype=torch.bfloat16, device="cuda")
    s = Setup(cached=[100, 7], fresh=[1, 90], q_heads=(0, 8), kv_heads=(0, 4), group=2, hd=hd, bt=bt, seed=4)
    big = arena.view(layers, 2, pool, n_kv, bt, hd)
    shift = pool - s.pool
    big[1, :, shift:].copy_(s.arena[0])
    t = np.where(s.table >= 0, s.table + shift, -1).astype(np.int32)
    s.d_table.copy_(torch.from_numpy(t))
    d = s.cache.d
    d.arena, d.arena_bytes, d.num_layers, d.num_blocks = arena.data_ptr(), arena.numel() * 2, layers, pool
    out, lse = s.attend(layer=1)
    s.check(out, lse)
    # and written there
    k = torch.randn(s.rows, n_kv, hd, device="cuda").to(torch.bfloat16)
    s.d_slots.copy_(torch.from_numpy(np.where(s.slots >= 0, s.slots + shift * bt, -1)))
    atp.kv_append(s.cache, s.step, 1, None, s.q.data_ptr(), s.q.stride(0), k.data_ptr(), k.stride(0), k.data_ptr(), k.stride(0),
                  out.data_ptr(), out.stride(0), stream())
    at = torch.from_numpy(s.slots + shift * bt).cuda()
    assert torch.equal(big[1, 1][at // bt, :, at % bt], k) and torch.equal(big[1, 0][at // bt, :, at % bt], k)


def test_attend_gives_the_same_bits_every_time():
    for kw in (dict(cached=[9000, 300], fresh=[1, 1]), dict(cached=[0, 900], fresh=[300, 200])):
        s = Setup(**kw, **GQA)
        a, la = s.attend()
        for _ in range(5):
            b, lb = s.attend()
            assert torch.equal(a, b) and torch.equal(la, lb)


# ---- atp_kv_extend ------------------------------------------------------------------

def run_extend(table, cached, fresh, bt, pool, max_tokens, in_place=False):
    table = np.asarray(table, np.int32)
    n, cols = table.shape
    d_table = dev(table, torch.int32)
    new = d_table if in_place else torch.full_like(d_table, 12345)
    guard = 64
    starts = torch.full((n + 1 + guard,), -9, dtype=torch.int32, device="cuda")
    slots = torch.full((max_tokens + guard,), -9, dtype=torch.int64, device="cuda")
    pos = torch.full((max_tokens + guard,), -9, dtype=torch.int32, device="cuda")
    status = torch.full((4,), -9, dtype=torch.int32, device="cuda")
    c, f = dev(cached, torch.int32), dev(fresh, torch.int32)
    cache = atp.KVCache(0, 0, 1, bt, 64, pool, (0, 0), (0, 0), 1)
    step = atp.KVStep(new.data_ptr(), n, cols, c.data_ptr(), f.data_ptr(), starts.data_ptr(), slots.data_ptr(), pos.data_ptr(),
                      max_tokens, 0, 0, status.data_ptr())
    need = atp.kv_extend_workspace(cache, step)
    ws = torch.full((need + 256,), 0xEE, dtype=torch.uint8, device="cuda")
    atp.kv_extend(cache, step, d_table.data_ptr(), ws.data_ptr(), need, stream())
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0xEE).all()) and bool((starts[n + 1:] == -9).all())
    assert bool((slots[max_tokens:] == -9).all()) and bool((pos[max_tokens:] == -9).all())
    return (new.cpu().numpy(), starts[:n + 1].tolist(), slots[:max_tokens].tolist(), pos[:max_tokens].tolist(), status.tolist())


def check_extend(table, cached, fresh, bt, pool, max_tokens):
    want = kvstep.extend(table, cached, fresh, bt, pool, max_tokens)
    for in_place in (False, True):
        got = run_extend(table, cached, fresh, bt, pool, max_tokens, in_place)
        assert np.array_equal(got[0], want[0]) and list(got[1:]) == list(want[1:]), (got[4], want[4])
    return want


def random_step(seed, n, cols, bt, pool, most_fresh, holes=0.0):
    rng = np.random.default_rng(seed)
    ids = iter(rng.permutation(pool).tolist())
    table, cached, fresh = np.full((n, cols), -1, np.int64), [], []
    for s in range(n):
        c = int(rng.integers(0, cols * bt + 1))
        f = int(rng.integers(0, min(most_fresh, cols * bt - c) + 1))
        for b in range(-(-c // bt) + int(rng.integers(0, 2))):
            if b < cols and rng.random() >= holes:
                table[s, b] = next(ids)
        cached.append(c)
        fresh.append(f)
    return table, cached, fresh


EXTEND = [  # n, cols, bt, pool, most_fresh
    (1, 1, 1, 1, 1), (1, 1, 16, 1, 16), (3, 4, 16, 16, 20), (8, 9, 16, 100, 1), (61, 33, 5, 4000, 3), (64, 40, 16, 2561, 200),
    (130, 17, 8, 2300, 40), (1, 5000, 16, 6000, 30000), (1100, 6, 4, 8000, 9), (40, 300, 16, 1_000_003, 2000), (300, 500, 1, 200_000, 50)]


@pytest.mark.parametrize("shape", EXTEND)
def test_extend(shape):
    n, cols, bt, pool, most = shape
    table, cached, fresh = random_step(n + cols, n, cols, bt, pool, most)
    w = check_extend(table, cached, fresh, bt, pool, sum(fresh) + 3)
    assert w[4][0] == 0


def test_extend_fills_holes_where_new_tokens_fall():
    table, cached, fresh = random_step(9, 30, 20, 8, 1200, 50, holes=0.3)
    assert check_extend(table, cached, fresh, 8, 1200, sum(fresh))[4][0] == 0


def test_extend_to_the_last_free_block_and_one_more():
    table = [[0, -1, -1], [3, -1, -1]]
    assert check_extend(table, [4, 2], [8, 6], 4, 5, 14)[4] == [0, 14, 3, 0]
    assert check_extend(table, [4, 2], [8, 7], 4, 5, 15)[4] == [atp.ECAPACITY, 0, 4, 3]
    assert check_extend(table, [4, 2], [8, 6], 4, 4, 14)[4] == [atp.ECAPACITY, 0, 3, 2]


@pytest.mark.parametrize("case", ["negative_cached", "negative_fresh", "past_table", "past_rows", "id_high", "id_low",
                                  "shared_written", "twice_in_a_row", "overflow"])
def test_extend_refuses_whole_steps(case):
    table, cached, fresh, rows = [[0, 1, -1], [2, -1, -1], [4, 5, -1]], [5, 2, 8], [1, 2, 1], 5
    if case == "negative_cached":
        cached[1] = -1
    elif case == "negative_fresh":
        fresh[1] = -1
    elif case == "past_table":
        fresh[2], rows = 5, 9
    elif case == "past_rows":
        rows = 3
    elif case == "id_high":
        table[1][2] = 9
    elif case == "id_low":
        table[1][2] = -2
    elif case == "shared_written":
        table[2][0] = 1
    elif case == "twice_in_a_row":
        table[0] = [1, 1, -1]
    else:
        cached[1], fresh[1] = 2 ** 31 - 1, 2 ** 31 - 1
    got = check_extend(table, cached, fresh, 4, 9, rows)
    assert got[4] == [atp.EINVAL, 0, 0, 0]


def test_extend_refuses_positions_past_31_bits():
    """A table wide enough for more than 2^31 - 1 tokens of a sequence (blocks of 2^26)."""
    table = [[-1] * 40]
    assert run_extend(table, [2 ** 31 - 2], [1], 1 << 26, 50, 1)[4][:2] == [0, 1]
    got = run_extend(table, [2 ** 31 - 2], [2], 1 << 26, 50, 2)
    assert got[4] == [atp.EINVAL, 0, 0, 0] and got[2] == [-1, -1] and np.array_equal(got[0], np.asarray(table))


def test_extend_keeps_shared_prefixes():
    table = [[7, 0, -1], [7, 1, -1], [7, -1, -1]]
    assert check_extend(table, [6, 8, 4], [2, 1, 3], 4, 9, 6)[4] == [0, 6, 2, 4]


def test_extend_with_no_sequence_and_no_token():
    assert check_extend(np.zeros((1, 2)) - 1, [0], [0], 4, 3, 0)[4] == [0, 0, 0, 3]
    assert check_extend(np.zeros((0, 2)), [], [], 4, 3, 2)[4] == [0, 0, 0, 3]


# ---- atp_kv_append ------------------------------------------------------------------

def run_append(s, layer=0, rope=None, in_place=False, offset=0):
    g = torch.Generator().manual_seed(11)
    n_q, n_kv, hd = s.n_q, s.n_kv, s.hd
    qkv = (2 * torch.randn(s.rows, (n_q + 2 * n_kv) * hd + offset, generator=g)).to(TORCH[s.dtype]).cuda()
    x = qkv[:, :(n_q + 2 * n_kv) * hd].double().cpu().numpy().reshape(s.rows, -1, hd)
    out = torch.full((s.rows, n_q * hd + offset), 7.0, dtype=TORCH[s.dtype], device="cuda")
    p, row = qkv.data_ptr(), qkv.stride(0)
    o, o_row = (p, row) if in_place else (out.data_ptr(), out.stride(0))
    before = qkv.clone()
    atp.kv_append(s.cache, s.step, layer, rope, p, row, p + 2 * n_q * hd, row, p + 2 * (n_q + n_kv) * hd, row, o, o_row, stream())
    torch.cuda.synchronize()
    got = qkv if in_place else out
    assert torch.equal(qkv[:, n_q * hd:], before[:, n_q * hd:]), "an input was written"
    if not in_place:
        assert torch.equal(qkv, before) and bool((out[:, n_q * hd:] == 7).all())
    return x, got[:, :n_q * hd].double().cpu().numpy().reshape(s.rows, n_q, hd), before[:, :n_q * hd].double().cpu().numpy().reshape(s.rows, n_q, hd)


def check_append(s, freqs, layer=0, rope=None, interleaved=False, amplitude=1.0, in_place=False, offset=0):
    before = s.heads_first(layer)
    x, q, q_in = run_append(s, layer, rope, in_place, offset)
    after, n_q, n_kv = s.heads_first(layer), s.n_q, s.n_kv
    real = s.slots >= 0
    turned = kvstep.rotate(x[:, :n_q + n_kv], s.positions, freqs, interleaved, amplitude)
    size = kvstep.rotate(np.abs(x[:, :n_q + n_kv]), np.zeros_like(s.positions), freqs, interleaved, amplitude)  # |x| * amplitude
    pair = np.zeros_like(size)
    n = len(freqs)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        pair[:, :, a] = pair[:, :, b] = size[:, :, a] + size[:, :, b]
    u = torch.finfo(TORCH[s.dtype]).eps / 2
    # cosine and sine off by 4 e, two products and a sum in 32 bits; then one rounding
    tol = u * np.abs(turned) + 8 * E * pair + (2.0 ** -25 if s.dtype == "fp16" else 0)
    assert np.all(np.abs(q - turned[:, :n_q])[real] <= tol[real][:, :n_q])
    assert np.array_equal(q[~real], (q_in if in_place else np.full_like(q, 7.0))[~real])
    want = np.concatenate([turned[:, n_q:], x[:, n_q + n_kv:]], 1)  # k heads, v heads
    ktol = np.concatenate([tol[:, n_q:], np.zeros_like(tol[:, n_q:])], 1)
    if s.e4m3:
        sc = s.scales[layer].double().cpu().numpy().reshape(-1)[None, :, None]
        lim = np.clip(want, -448 * sc, 448 * sc)
        err32 = np.concatenate([8 * E * pair[:, n_q:], np.zeros_like(pair[:, n_q:])], 1) + 2 * E * np.abs(want)
        ktol = 2.0 ** -4 * np.abs(lim) + 2.0 ** -10 * sc + 2 * err32
        want = lim
    for t in np.flatnonzero(real):
        p, o = divmod(int(s.slots[t]), s.bt)
        for w in range(2):
            d = np.abs(after[w, p, :, o] - want[t, w * n_kv:(w + 1) * n_kv])
            assert np.all(d <= ktol[t, w * n_kv:(w + 1) * n_kv]), (t, w, float(d.max()))
            before[w, p, :, o] = after[w, p, :, o]
    assert np.array_equal(before, after, equal_nan=True), "something else of the cache was written"


APPEND = {
    "one": dict(cached=[0], fresh=[1]),
    "tiny": dict(cached=[127, 0, 15, 3], fresh=[1, 1, 1, 1], q_heads=(0, 2), group=2, hd=64, dtype="fp16", pad=3),
    "prompt": dict(cached=[3, 70000], fresh=[40, 19], **GQA),
    "token_major": dict(cached=[3, 70], fresh=[40, 1], layout="token", bt=8, pad=1, **GQA),
    "e4m3": dict(cached=[3, 70], fresh=[40, 1], cache="e4m3", **GQA),
    "e4m3_token_fp16": dict(cached=[3, 70], fresh=[9, 1], cache="e4m3", layout="token", dtype="fp16", **GQA),
    "dim_72": dict(cached=[9], fresh=[20], hd=72, bt=5, q_heads=(1, 6), kv_heads=(0, 2), group=4),
    "dim_8": dict(cached=[9], fresh=[3], hd=8, q_heads=(1, 6), kv_heads=(0, 2), group=4),
    "dim_256": dict(cached=[9], fresh=[20], hd=256, q_heads=(1, 6), kv_heads=(0, 2), group=4),
    "layers": dict(cached=[9], fresh=[20], layers=3, **GQA),
    "kv_only": dict(cached=[9], fresh=[20], q_heads=(4, 4), kv_heads=(0, 2), group=2),
}


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("part", ["whole", "half", "odd", "none"])
@pytest.mark.parametrize("name", APPEND)
def test_append(name, part, interleaved):
    s = Setup(**APPEND[name])
    rot = {"whole": s.hd, "half": s.hd // 2, "odd": max(2, s.hd // 2 - 2), "none": 0}[part]
    check_append(s, kvstep.frequencies(rot, 10000.0), s.layers - 1, atp.Rope(rot, interleaved=interleaved) if rot else None, interleaved)


@pytest.mark.parametrize("scaling", ["linear", "parts"])
def test_append_scaled_positions(scaling):
    kw = dict(factor=8.0, low=1.0, high=32.0, original=4096.0) if scaling == "parts" else dict(factor=3.0)
    s = Setup(cached=[0, 100000], fresh=[30, 30], **GQA)
    rope = atp.Rope(128, 500000.0, scaling=atp.ROPE_PARTS if scaling == "parts" else atp.ROPE_LINEAR, amplitude=1.25, **kw)
    check_append(s, kvstep.frequencies(128, 500000.0, scaling, **kw), rope=rope, amplitude=1.25)


def test_append_far_positions_keep_their_phase():
    s = Setup(cached=[5], fresh=[4], **GQA)
    s.positions = np.array([2 ** 31 - 1, 2 ** 24 + 1, 12345678, 1], np.int32)
    s.d_pos.copy_(torch.from_numpy(s.positions))
    check_append(s, kvstep.frequencies(128, 10000.0), rope=atp.Rope(128))


@pytest.mark.parametrize("in_place", [False, True])
def test_append_in_place_and_wide_rows(in_place):
    s = Setup(cached=[5, 0], fresh=[40, 3], pad=2, **GQA)
    check_append(s, kvstep.frequencies(128, 10000.0), rope=atp.Rope(128), in_place=in_place, offset=24)


def test_append_e4m3_saturates_and_keeps_nan():
    s = Setup(cached=[0], fresh=[2], cache="e4m3", q_heads=(0, 1), group=1, hd=64)
    s.scales.fill_(1.0)
    row = torch.tensor([449.0, 1e30, math.inf, -449.0, -math.inf, math.nan, 448.0, -0.0, 2.0 ** -10, 2.0 ** -9, 1.5 * 2.0 ** -9, 465.0]
                       + [0.0] * 52, dtype=torch.bfloat16, device="cuda").repeat(2, 1)
    out = torch.empty_like(row)
    atp.kv_append(s.cache, s.step, 0, None, row.data_ptr(), 64, row.data_ptr(), 64, row.data_ptr(), 64, out.data_ptr(), 64, stream())
    p, o = divmod(int(s.slots[1]), 16)
    for w in range(2):
        got = s.arena[0, w, p, 0, o, :12].float().tolist()
        assert got[:5] == [448.0, 448.0, 448.0, -448.0, -448.0] and math.isnan(got[5])
        assert got[6:] == [448.0, 0.0, 0.0, 2.0 ** -9, 2.0 ** -8, 448.0] and math.copysign(1, got[7]) == -1
    assert torch.equal(out.view(torch.int16), row.view(torch.int16))


def test_append_reports_slots_past_the_arena():
    s = Setup(cached=[0], fresh=[3], pool_extra=0, **GQA)
    s.slots[1] = s.pool * s.bt
    s.d_slots.copy_(torch.from_numpy(s.slots))
    before = s.heads_first()
    x, q, _ = run_append(s, rope=None)
    assert s.status.tolist()[0] == atp.EINVAL
    assert np.array_equal(q, x[:, :s.n_q])  # q of that token too
    s.slots[1] = -1
    after = s.heads_first()
    for t in (0, 2):
        before[:, s.slots[t] // s.bt, :, s.slots[t] % s.bt] = after[:, s.slots[t] // s.bt, :, s.slots[t] % s.bt]
    assert np.array_equal(before, after)

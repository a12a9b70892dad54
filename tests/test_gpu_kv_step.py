"""The KV cache operators as a serving loop uses them: on the arena a reshard
leaves, step after step, captured into a HIP graph, and on several streams."""
import numpy as np
import pytest
import torch

from oracle import kvstep
from paper_2511_11617_amd import atp, problem
from synth import configs
from tests.gpu_harness import prepare_case
from tests.test_gpu_kv_ops import E, TORCH, Setup, dev, stream

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


class Loop:
    """A serving loop over one layer's arena: places, rotation and cache write,
    attention, with the buffers a program keeps."""

    def __init__(self, arena, pool, table, q_heads, kv_heads, group, hd, bt, dtype, layout, rows, max_fresh, max_ctx, layers=1):
        self.dt, self.hd, self.bt, self.pool, self.rows, self.layers = TORCH[dtype], hd, bt, pool, rows, layers
        self.q_heads, self.kv_heads, self.group = q_heads, kv_heads, group
        self.n_q, self.n_kv = q_heads[1] - q_heads[0], kv_heads[1] - kv_heads[0]
        n, cols = table.shape
        self.arena, self.table = arena, dev(table, torch.int32)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.cached, self.fresh, self.starts = torch.zeros(n, **i32), torch.zeros(n, **i32), torch.zeros(n + 1, **i32)
        self.slots, self.pos = torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.zeros(rows, **i32)
        self.status = torch.zeros(4, **i32)
        self.qkv = torch.zeros(rows, (self.n_q + 2 * self.n_kv) * hd, dtype=self.dt, device="cuda")
        self.q = torch.zeros(rows, self.n_q, hd, dtype=self.dt, device="cuda")
        self.out = torch.zeros_like(self.q)
        self.lse = torch.zeros(rows, self.n_q, device="cuda")
        self.cache = atp.KVCache(arena.data_ptr(), arena.numel() * arena.element_size(), layers, bt, hd, pool, q_heads, kv_heads,
                                 group, atp.BF16 if dtype == "bf16" else atp.FP16,
                                 layout=atp.KV_HEAD_MAJOR if layout == "head" else atp.KV_TOKEN_MAJOR)
        self.step = atp.KVStep(self.table.data_ptr(), n, cols, self.cached.data_ptr(), self.fresh.data_ptr(), self.starts.data_ptr(),
                               self.slots.data_ptr(), self.pos.data_ptr(), rows, max_fresh, max_ctx, self.status.data_ptr())
        self.rope, self.mask = atp.Rope(hd), atp.Mask(hd ** -0.5)
        self.n_ext, self.n_att = atp.kv_extend_workspace(self.cache, self.step), atp.kv_attend_workspace(self.cache, self.step)
        self.ws = torch.empty(self.n_ext + self.n_att + 512, dtype=torch.uint8, device="cuda")

    def run(self, layer=0, s=None):
        s = stream() if s is None else s
        p, row, hd = self.qkv.data_ptr(), self.qkv.stride(0), self.hd
        atp.kv_extend(self.cache, self.step, self.table.data_ptr(), self.ws.data_ptr(), self.n_ext, s)
        atp.kv_append(self.cache, self.step, layer, self.rope, p, row, p + 2 * self.n_q * hd, row,
                      p + 2 * (self.n_q + self.n_kv) * hd, row, self.q.data_ptr(), self.q.stride(0), s)
        ws = self.ws.data_ptr() + (self.n_ext + 255) // 256 * 256
        atp.kv_attend(self.cache, self.step, layer, self.mask, self.q.data_ptr(), self.q.stride(0), self.out.data_ptr(),
                      self.out.stride(0), self.lse.data_ptr(), ws, self.n_att, s)

    def expect(self, keys, values, qkv, cached, fresh):
        """The 64-bit result, from the contexts' rotated K and V (in the cache's
        precision) before the step; extends them."""
        n_q, n_kv, hd = self.n_q, self.n_kv, self.hd
        starts = np.concatenate([[0], np.cumsum(fresh)])
        pos = np.concatenate([np.arange(c, c + f) for c, f in zip(cached, fresh)]).astype(int)
        x = qkv[:len(pos)].reshape(len(pos), -1, hd)
        turned = kvstep.rotate(x[:, :n_q + n_kv], pos, kvstep.frequencies(hd, 10000.0))
        low = lambda y: torch.from_numpy(y).to(self.dt).double().numpy()  # noqa: E731
        q, k, v = low(turned[:, :n_q]), low(turned[:, n_q:]), x[:, n_q + n_kv:]
        for s in range(len(fresh)):
            keys[s] = np.concatenate([keys[s], k[starts[s]:starts[s + 1]]])
            values[s] = np.concatenate([values[s], v[starts[s]:starts[s + 1]]])
        return kvstep.attend(q, keys, values, starts.tolist(), cached, self.q_heads, self.kv_heads, self.group, hd ** -0.5), len(pos)

    def check(self, want, rows):
        (out, lse, weight, reach), u = want, torch.finfo(self.dt).eps / 2
        # q and k: one rounding each may fall the other way (their 32-bit rotation is off by some e), so a score is off
        # by 2 u of its products; then as for the attention alone
        ds = (2 * u + (self.hd + 24) * E) * reach
        tol = u * np.abs(out) + 1.1 * weight * (u + 2 * ds[..., None] + 4096 * E) + 2.0 ** -24
        got = self.out[:rows].double().cpu().numpy()
        assert np.all(np.abs(got - out) <= tol), float((np.abs(got - out) / tol).max())
        assert np.all(np.abs(self.lse[:rows].double().cpu().numpy() - lse) <= ds + 4096 * E + 8 * E * np.abs(lse))


@pytest.mark.parametrize("layout", ["head", "token"])
def test_serving_goes_on_after_a_reshard(layout):
    """A TP 4 -> 3 reshard on the GPU, then on its arena, its table and its head
    ranges: a step of one token each, a step with drafts, and a prompt in a
    new row of the table; every step against the 64-bit oracle over the
    contexts that the full cache defines."""
    c = configs.get(1, hidden=512, n_q=12, n_kv=4, head_dim=64, new_q_widths=[5, 4, 3], new_ffn_widths=None, self_old=2, n_seq=6,
                    seq_tokens=112, kv_layout=layout, fragmented=True, pool_factor=2.0)
    finish = prepare_case(c, name=f"serve-{layout}")()
    finish()
    arena, table = finish.keep[3], finish.keep[10].cpu().numpy()
    plan = problem.build(c).plan()
    me = plan.stats().self_new_rank
    q_heads, kv_heads = plan.ranges(problem.SPACE_Q)[me], plan.ranges(problem.SPACE_KV)[me]
    assert q_heads == (5, 9) and kv_heads == (1, 3)  # begins inside the second group of 3
    layers, bt, hd, n_kv = c["layers"], c["block_tokens"], 64, 2
    pool = int(2 * 6 * 7)
    size = layers * 2 * pool * n_kv * bt * hd
    arena = arena[:size * 2].view(torch.float16)
    shape = (layers, 2, pool, n_kv, bt, hd) if layout == "head" else (layers, 2, pool, bt, n_kv, hd)
    a = arena.view(shape).double().cpu().numpy()
    a = a if layout == "head" else a.transpose(0, 1, 2, 4, 3, 5)
    wide = np.full((7, 20), -1, np.int32)
    wide[:6, :table.shape[1]] = table
    t = np.arange(112)
    keys = [[a[l, 0][table[s, t // bt], :, t % bt] for s in range(6)] + [np.zeros((0, n_kv, hd))] for l in range(layers)]
    values = [[a[l, 1][table[s, t // bt], :, t % bt] for s in range(6)] + [np.zeros((0, n_kv, hd))] for l in range(layers)]
    loop = Loop(arena, pool, wide, q_heads, kv_heads, 3, hd, bt, "fp16", layout, 80, 64, 192, layers)
    cached = [112] * 6 + [0]
    g = torch.Generator().manual_seed(3)
    for fresh in ([1] * 6 + [0], [2, 0, 3, 1, 1, 4, 0], [1, 1, 0, 1, 1, 1, 61], [1] * 7):
        loop.cached.copy_(torch.tensor(cached))
        loop.fresh.copy_(torch.tensor(fresh))
        for l in range(layers):
            loop.qkv.copy_(torch.randn(loop.qkv.shape, generator=g).to(torch.float16))
            loop.run(l)
            torch.cuda.synchronize()
            assert loop.status.tolist()[:2] == [0, sum(fresh)]
            want, rows = loop.expect(keys[l], values[l], loop.qkv.double().cpu().numpy(), cached, fresh)
            loop.check(want, rows)
        cached = [x + f for x, f in zip(cached, fresh)]


def fresh_loop(n=5, cols=80, max_fresh=1, rows=8, seed=0, max_ctx=1200):
    pool = 300
    g = torch.Generator().manual_seed(seed)
    arena = torch.randn(1, 2, pool, 2, 16, 128, generator=g).to(torch.bfloat16).cuda()
    ids = np.random.default_rng(seed).permutation(pool)
    table = np.full((n, cols), -1, np.int32)
    table[:, :50] = ids[:n * 50].reshape(n, 50)
    return Loop(arena, pool, table, (10, 19), (1, 3), 8, 128, 16, "bf16", "head", rows, max_fresh, max_ctx)


@pytest.mark.parametrize("max_fresh", [1, 40])
def test_a_captured_step_replays_with_other_lengths(max_fresh):
    """One captured step, replayed over steps whose lengths the device holds,
    between eager work and synchronizations, equals the eager steps bit for
    bit; two graphs that share a workspace run one after the other."""
    rows = 8 if max_fresh == 1 else 64
    eager, a = fresh_loop(max_fresh=max_fresh, rows=rows), fresh_loop(max_fresh=max_fresh, rows=rows)
    first = eager.table.clone()
    a.run()  # the kernels are loaded before a capture
    a.table.copy_(first)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        s = torch.cuda.Stream()
        with torch.cuda.graph(g, stream=s):
            a.run(s=s.cuda_stream)
            a.cached.add_(a.fresh)
        graphs.append(g)
    gen = torch.Generator().manual_seed(5)
    for loop in (eager, a):
        loop.cached.copy_(torch.tensor([800, 1, 333, 16, 47]))
    eager.arena.copy_(a.arena)
    for i in range(6):
        fresh = [1, 1, 0, 1, 1] if max_fresh == 1 else [[1, 40, 0, 3, 1], [2, 0, 17, 1, 30], [0, 0, 0, 0, 0]][i % 3]
        x = torch.randn(a.qkv.shape, generator=gen).to(torch.bfloat16)
        for loop in (eager, a):
            loop.fresh.copy_(torch.tensor(fresh))
            loop.qkv.copy_(x)
        eager.run()
        eager.cached.add_(eager.fresh)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        for name in ("out", "lse", "table", "slots", "pos", "starts", "cached", "status"):
            assert torch.equal(getattr(eager, name), getattr(a, name)), (i, name)
        assert torch.equal(eager.arena, a.arena)
        torch.zeros(1 << 20, device="cuda").sum()  # other work between the replays


def test_steps_on_two_streams_at_once():
    """Two loops with buffers of their own on two streams, neither of them the
    current one, give what each gives alone."""
    loops = [fresh_loop(seed=s, max_fresh=40, rows=64) for s in (1, 2)]
    alone = [fresh_loop(seed=s, max_fresh=40, rows=64) for s in (1, 2)]
    g = torch.Generator().manual_seed(9)
    for a, b in zip(loops, alone):
        x = torch.randn(a.qkv.shape, generator=g).to(torch.bfloat16)
        for loop in (a, b):
            loop.cached.copy_(torch.tensor([700, 20, 333, 0, 47]))
            loop.fresh.copy_(torch.tensor([1, 40, 1, 17, 2]))
            loop.qkv.copy_(x)
    for b in alone:
        b.run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for a, s in zip(loops, streams):
            a.run(s=s.cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(loops, alone):
        assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse) and torch.equal(a.arena, b.arena)


def test_a_refused_step_does_nothing():
    """After a refused extend (no blocks left), append and attend of the step
    touch nothing."""
    loop = fresh_loop(max_fresh=40, rows=64)
    loop.cached.copy_(torch.tensor([800, 800, 800, 800, 800]))
    loop.fresh.copy_(torch.tensor([40, 24, 0, 0, 0]))
    loop.table[0, 50:60] = torch.arange(10, dtype=torch.int32, device="cuda")  # ids of other rows: shared blocks
    before, out = loop.arena.clone(), loop.out.clone()
    loop.run()
    torch.cuda.synchronize()
    assert loop.status.tolist()[0] == atp.EINVAL
    assert torch.equal(loop.arena, before) and torch.equal(loop.out, out)


def test_setup_matches_the_cache_layout():
    """The two layouts hold the same values at the same places (the helper the other tests lean on)."""
    s = Setup(cached=[5], fresh=[2], q_heads=(0, 2), kv_heads=(0, 2), group=1, hd=16, layout="token")
    a = s.heads_first()
    assert a.shape == (2, s.pool, 2, 16, 16)
    assert a[1, 3, 1, 7, 5] == float(s.arena[0, 1, 3, 7, 1, 5])

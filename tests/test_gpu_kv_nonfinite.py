"""Infinities and NaN that rows see in V (GPU, through the C ABI): each makes
its dimension of those rows that value, whatever its weight, and changes
nothing else by a bit."""
import math

import pytest
import torch

from tests.test_gpu_kv_ops import GQA, Setup

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


SHAPES = {
    "one_chunk": dict(cached=[250], fresh=[1]),                     # a step or two a wave, no split
    "split": dict(cached=[2000], fresh=[1]),                        # chunks of 256, joined
    "split_token_major": dict(cached=[2000, 600], fresh=[1, 1], layout="token"),
    "blocks_of_5": dict(cached=[700], fresh=[1], bt=5),
    "dim_80": dict(cached=[700], fresh=[1], hd=80),
    "dim_256": dict(cached=[700], fresh=[1], hd=256),
    "drafts": dict(cached=[2000], fresh=[4]),
    "long_chunk": dict(cached=[6000] * 64, fresh=[1] * 64),         # several steps a wave
    "prompt": dict(cached=[0], fresh=[300]),
    "prompt_cut": dict(cached=[2000], fresh=[40]),                  # tiles in parts, joined
    "prompt_64_token_major": dict(cached=[600], fresh=[90], hd=64, layout="token"),
    "prompt_80": dict(cached=[600], fresh=[70], hd=80),
    "prompt_256": dict(cached=[600], fresh=[70], hd=256),
}
CASES = [(n, t, c) for n in SHAPES for t in ("bf16", "fp16") for c in ("same", "e4m3")]


# "sharp": scores spread over hundreds, so most weights are 0 in 32 bits, whole chunks' among them
@pytest.mark.parametrize("scale", ["usual", "sharp"])
@pytest.mark.parametrize("name,dtype,cache", CASES)
def test_attend_non_finite_values_that_are_seen(name, dtype, cache, scale):
    s = Setup(**SHAPES[name], **GQA, dtype=dtype, cache=cache, seed=21)
    ctx, q = s.cached[0] + s.fresh[0], 0
    m = dict(scale=s.hd ** -0.5 if scale == "usual" else 8.0)
    a = s.arena.view(torch.uint8) if s.e4m3 else s.arena

    def put(t, d, x):  # at token t of the first sequence, in the first KV head's V
        p, o = int(s.table[q, t // s.bt]), t % s.bt
        at = (0, 1, p, 0, o, d) if s.layout == "head" else (0, 1, p, o, 0, d)
        a[at] = x

    # (token, dimension, value): the first, a middle and the last step, and one infinity of each sign
    nan = 0x7F if s.e4m3 else math.nan
    wild = [(t, 3 * i + 2, nan) for i, t in enumerate((0, ctx // 2, ctx - 1))]
    if not s.e4m3:
        wild += [(t, 3 * i + 0, math.inf) for i, t in enumerate((0, ctx // 2, ctx - 1))]
        wild += [(t, 3 * i + 1, -math.inf) for i, t in enumerate((0, ctx // 2, ctx - 1))]
        wild += [(7, s.hd - 1, math.inf), (ctx // 3, s.hd - 1, -math.inf), (9, s.hd - 2, math.inf), (ctx // 3, s.hd - 2, math.inf)]
    for t, d, _ in wild:
        put(t, d, 0)
    calm, calm_lse = s.attend(**m)
    if name != "long_chunk":  # the oracle takes its time over 64 contexts
        s.check(calm, calm_lse, **m)
    for t, d, x in wild:
        put(t, d, x)
    want = calm.clone()
    pos = s.cached[0] + torch.arange(s.fresh[0])
    first = 6  # query heads 10 to 15 read KV head 1, the first of the range
    for t, d, x in wild:
        rows = torch.nonzero(pos >= t).flatten().cuda()
        want[rows, :first, d] += math.nan if s.e4m3 else x
    out, lse = s.attend(**m)
    assert torch.equal(torch.isnan(out), torch.isnan(want)), int((torch.isnan(out) != torch.isnan(want)).sum())
    assert torch.equal(torch.nan_to_num(out, nan=5.0), torch.nan_to_num(want, nan=5.0)) and torch.equal(lse, calm_lse)
    assert s.status.tolist()[0] == 0


@pytest.mark.parametrize("shape", ["split", "prompt_cut"])
def test_attend_non_finite_values_before_a_window(shape):
    """The same with a window: rows whose window has passed the value keep it out."""
    s = Setup(**SHAPES[shape], **GQA, seed=22)
    t, window = s.cached[0] - 300, 310
    calm, _ = s.attend(window=window)
    p, o = int(s.table[0, t // 16]), t % 16
    s.arena[0, 1, p, 0, o, 3] = math.inf
    sees = torch.nonzero(s.cached[0] + torch.arange(s.fresh[0]) - t < window).flatten().cuda()
    assert 0 < len(sees) < 40
    out, _ = s.attend(window=window)
    calm[sees, :6, 3] = math.inf
    assert torch.equal(out, calm)

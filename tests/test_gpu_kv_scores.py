"""atp_kv_attend where a row's scores are -infinity (K holds one against the
query's sign): such a token weighs nothing, and a row of them alone is as one
that sees nothing.  GPU, through the C ABI."""
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


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", [dict(cached=[100], fresh=[1]), dict(cached=[2000], fresh=[3]), dict(cached=[200], fresh=[80])])
def test_scores_of_minus_infinity(shape, dtype):
    s = Setup(**shape, **GQA, dtype=dtype, seed=41)
    s.q[..., 0] = s.q[..., 0].abs() + 0.5
    calm_k = s.arena.clone()
    # tokens of the first KV head's blocks 0 and 2 have the score -infinity: as if the blocks were absent
    t = s.table.copy()
    for b in (0, 2):
        s.arena[0, 0, int(t[0, b]), 0, :, 0] = -math.inf
    out, lse = s.attend()
    gone = t.copy()
    gone[0, [0, 2]] = -1
    s.arena.copy_(calm_k)
    s.d_table.copy_(torch.from_numpy(gone))
    want, want_lse = s.attend()
    assert torch.equal(out[:, :6], want[:, :6]) and torch.equal(lse[:, :6], want_lse[:, :6])  # the heads that read it
    # every one of its tokens: nothing is left for those heads
    s.d_table.copy_(torch.from_numpy(t))
    s.arena[0, 0, :, 0, :, 0] = -math.inf
    out, lse = s.attend()
    assert bool((out[:, :6] == 0).all()) and bool(torch.isneginf(lse[:, :6]).all())
    assert bool(torch.isfinite(lse[:, 6:]).all()) and bool(torch.isfinite(out).all())

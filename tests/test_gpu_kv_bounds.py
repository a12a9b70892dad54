"""KV cache operators with bounds far above the lengths, as a captured step has
them (GPU, through the C ABI)."""
import pytest
import torch

from paper_2511_11617_amd import atp
from tests.test_gpu_kv_ops import Setup, stream

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("max_ctx", [1300, 1 << 17, 1 << 30])
def test_the_list_of_prompt_tiles_goes_from_long_to_short_whatever_the_bound(max_ctx):
    """The list is the workspace's begin: 12 words an item (sequence, run, tile,
    first token, last token + 1, ...; sequence -1: none).  Its order is by 32
    classes of the longest item."""
    s = Setup(cached=[0, 40, 3, 0], fresh=[1300, 700, 900, 200], q_heads=(0, 48), kv_heads=(0, 3), group=16, hd=64, bounds=(1300, max_ctx))
    need = atp.kv_attend_workspace(s.cache, s.step)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(s.q)
    atp.kv_attend(s.cache, s.step, 0, atp.Mask(s.hd ** -0.5), s.q.data_ptr(), s.q.stride(0), out.data_ptr(), out.stride(0), 0,
                  ws.data_ptr(), need, stream())
    torch.cuda.synchronize()
    tiles = sum(-(-f * 16 // 128) for f in s.fresh) * 3
    items = ws[:need // 48 * 48].view(torch.int32).reshape(-1, 12)[:tiles].cpu()
    assert bool((items[:, 0] >= 0).all()) and sorted(set(items[:, 0].tolist())) == [0, 1, 2, 3]
    span = items[:, 4] - items[:, 3]
    longest = int(span.max())
    assert longest == 1300
    after = span.flip(0).cummax(0).values.flip(0)  # the longest from each place on
    assert bool((after <= span + 64 + longest // 32).all())  # spans are rounded up to 64 tokens
    assert s.status.tolist()[0] == 0

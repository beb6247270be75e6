"""Attention with upper bounds of the lengths far above the lengths themselves, as in steps whose sizes are captured once."""
import pytest

from tests.gpu_util import announce, torch_cuda
from tests.test_gpu_ops import A, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [4, 32])
def test_loose_bounds(dtype, dim):
    """64 sequences of 80 heads under bounds of 2^20 rows: more than 2^32 rows of scores if all were there."""
    torch = torch_cuda()
    announce(f"attention with bounds of 2^20 {dtype} {dim}")
    c = Case(dtype=dtype, lens=tuple((3 + i % 38, 40 - i % 37) for i in range(64)), heads=80, dim=dim, mask=1, gap=1, seed=90)
    c.a.max_q = c.a.max_k = 1 << 20
    c.ws = torch.full((A.fo_attn_workspace(c.a, True),), 0xFF, dtype=torch.uint8, device="cuda")
    c.run()
    torch.cuda.synchronize()
    c.verify()

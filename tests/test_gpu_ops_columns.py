"""Dropout of a row of more than 2^27 columns: the last step of its bias gradient has a workgroup for 32 of them."""
import pytest

from tests.gpu_util import announce, torch_cuda

pytestmark = pytest.mark.gpu
A = pytest.importorskip("paper_2504_13850_amd.api")


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_bias_gradient_of_many_columns(dtype):
    """A single row: the bias gradient is dx itself, bit for bit."""
    torch = torch_cuda()
    cols = (1 << 27) + 40
    announce(f"dropout of {cols} columns {dtype}")
    g = torch.Generator(device="cuda").manual_seed(1)
    dy = torch.randn((1, cols), generator=g, device="cuda", dtype=torch.float32).to(getattr(torch, dtype))
    dx, dbias = torch.empty_like(dy), torch.full((cols,), float("nan"), dtype=dy.dtype, device="cuda")
    ws = torch.empty(A.fo_dropout_workspace(1, cols), dtype=torch.uint8, device="cuda")
    A.fo_dropout_bwd(dy, dx, 0.25, 3, 4, dbias=dbias, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(dx[0], dbias)
    share = float((dx == 0).float().mean())
    assert abs(share - 0.25) <= 1e-3

"""Attention whose scores all lie several caps below zero, or above: the softmax is over what is left of their
differences, and cap tanh has to be as good there as fp32 holds it (a cap of 200 times 2^-25: 6e-6, below the 2^-18 and
its factor of two that test_gpu_ops asks of fp32).  The forward pass only: the backward one starts from lse, here 288 in
base 2, whose own rounding in fp32 is up to 1e-5 of every probability of a row."""
import pytest

from tests.gpu_util import announce, torch_cuda
from tests.test_gpu_ops import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("kw", [
    dict(lens=((200, 200), (70, 150)), heads=4, kv_heads=2, dim=64), dict(lens=((100, 100), (40, 128)), heads=3, dim=32),
    dict(lens=((200, 200), (70, 150)), heads=4, kv_heads=2, dim=4), dict(lens=((1, 3000),), heads=4, kv_heads=1, dim=64)],
    ids=["tiled", "short", "narrow", "one"])
def test_scores_far_beyond_the_cap(dtype, sign, kw):
    torch = torch_cuda()
    announce(f"attention, scores of {sign * 4} caps {dtype} {kw}")
    c = Case(dtype=dtype, cap=200.0, seed=600, train=False, **kw)
    d = kw["dim"]
    c.q.mul_(0.1).add_(1.0)
    c.k.mul_(0.1).add_(1.0).mul_(sign * 800.0 / d ** 0.5)  # scale q.k: about 800, by 0.14 / sqrt(d) of it more or less
    c.run()
    c.verify()

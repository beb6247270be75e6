"""Attention under scales far from one: queries and keys 2^50 times as large and a scale of 2^-100 times are the same
scores, and powers of two round nowhere, so that every result has the same bits but for its exponent."""
import pytest

from tests.gpu_util import announce, torch_cuda
from tests.test_gpu_ops import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [
    dict(lens=((200, 200), (70, 150)), heads=4, kv_heads=2, dim=64, mask=1), dict(lens=((60, 60),), heads=2, dim=32, mask=1, radius=9),
    dict(lens=((300, 200),), heads=2, kv_heads=1, dim=128, cap=4.0, p=0.1), dict(lens=((100, 100),), heads=3, dim=4, mask=1),
    dict(lens=((1, 3000),), heads=4, kv_heads=1, dim=64, train=False), dict(lens=((200, 200),), heads=2, dim=77, layout="odd")],
    ids=lambda k: "-".join(f"{n}{v}" for n, v in k.items()).replace(" ", ""))
def test_powers_of_two(dtype, kw):
    torch = torch_cuda()
    announce(f"attention scaled by powers of two {dtype} {kw}")
    big, small = 2.0 ** 50, 2.0 ** -100
    a, b = (Case(dtype=dtype, scale=s, seed=70, **kw) for s in (0.125, 0.125 * small))
    b.q.mul_(big)
    b.k.mul_(big)
    a.run()
    b.run()
    torch.cuda.synchronize()
    a.verify()
    if a.train:
        for t in b.grads[:2]:
            t.mul_(big)
        assert torch.equal(a.lse.nan_to_num(7.0), b.lse.nan_to_num(7.0))
    for x, y in zip(a.outputs(), b.outputs()):
        assert torch.equal(x.isnan(), y.isnan()) and torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))

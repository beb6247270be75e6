"""Forms of the attention at sizes that reach each of its kernels: the tiled ones (long sequences or shared key heads), the
short one (up to 128 rows) and those of narrow heads."""
import pytest

from tests.gpu_util import announce, torch_cuda
from tests.test_gpu_ops import Case, check

pytestmark = pytest.mark.gpu
TILED = dict(lens=((200, 200), (70, 150)), heads=4, kv_heads=2, dim=64)
SHORT = dict(lens=((100, 100), (1, 1), (40, 128)), heads=3, dim=32)
NARROW = dict(lens=((200, 200), (1, 1), (70, 150)), heads=4, kv_heads=2, dim=4)
KERNELS = pytest.mark.parametrize("kw", [TILED, SHORT, NARROW], ids=["tiled", "short", "narrow"])
DTYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])


@KERNELS
@DTYPES
@pytest.mark.parametrize("cap", [0.0, 2.0])
@pytest.mark.parametrize("scale", [-0.3, 0.0])
def test_negative_and_zero_scale(kw, dtype, cap, scale):
    check(dtype=dtype, mask=1, cap=cap, scale=scale, radius=8, p=0.1, seed=500, **kw)


@KERNELS
@DTYPES
@pytest.mark.parametrize("hide", ["inf", "lowest"])
def test_hidden_distances(kw, dtype, hide):
    check(dtype=dtype, mask=1, radius=30, n_buckets=3, hide=hide, seed=501, **kw)


@KERNELS
@DTYPES
def test_all_distances_hidden(kw, dtype):
    """A table that hides every key: results and gradients of zero."""
    torch = torch_cuda()
    announce(f"attention, everything hidden {dtype} {kw}")
    c = Case(dtype=dtype, radius=30, n_buckets=3, seed=502, **kw)
    c.table.fill_(-float("inf"))
    c.run()
    torch.cuda.synchronize()
    c.verify()
    for lo, hi, klo, khi in c.spans:
        assert not c.out[lo:hi].any() and not any(g[klo:khi].any() for g in c.grads[1:])


@KERNELS
@DTYPES
def test_bounds_are_clamped(kw, dtype):
    """Bounds outside the rows or reversed reach no row that is not there."""
    torch = torch_cuda()
    announce(f"attention with bounds out of range {dtype} {kw}")
    n = kw["lens"][0][0]
    c = Case(dtype=dtype, mask=1, radius=5, seed=503, **{**kw, "lens": ((n, n), (30, 30), (90, 90))})
    on = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    keep = [on(-5, n + 60, n + 30), on(n, n + 40, 2000000000), on(-5, n + 60, n + 30), on(n, n + 40, 2000000000)]
    for name, t in zip(("q_begin", "q_end", "k_begin", "k_end"), keep):
        setattr(c.a, name, t.data_ptr())
    c.run()
    c.spans = [(0, n, 0, n), (n + 60,) * 2 + (n + 60,) * 2, (n + 30, n + 120, n + 30, n + 120)]
    torch.cuda.synchronize()
    c.verify()


@DTYPES
@pytest.mark.parametrize("keys", [60, 3000])
def test_nan_query_of_a_narrow_head(dtype, keys):
    """Its own result is not a number, and the other rows' are as without it, but for the last bits: rows of a wave move
    their running maximum together."""
    torch = torch_cuda()
    announce(f"narrow attention with a NaN query {dtype} {keys}")
    c = Case(dtype=dtype, lens=((40, keys),), heads=4, kv_heads=2, dim=4, train=False, seed=504)
    c.run()
    torch.cuda.synchronize()
    want = c.out.clone()
    c.q[39, 1] = float("nan")
    c.run()
    torch.cuda.synchronize()
    assert torch.isnan(c.out[39, 1]).all()
    want[39, 1] = c.out[39, 1] = 0
    eps = {"bf16": 2.0 ** -7, "f32": 2.0 ** -18}[dtype]  # two roundings of a result; sums in another order
    assert float((c.out - want).abs().max()) <= eps * float(want.abs().max())


@KERNELS
@DTYPES
def test_capped_scores_of_several_caps(kw, dtype):
    """Scores whose spread is several caps, so that most of them are held by the cap, and a cap of thousands."""
    check(dtype=dtype, mask=1, cap=50.0, scale=20.0, seed=505, **kw)
    check(dtype=dtype, mask=1, cap=1000.0, scale=0.125, seed=506, **kw)


@DTYPES
@pytest.mark.parametrize("lens,kv", [(((20, 300), (32, 5)), 1), (((130, 40), (64, 64)), 2), (((300, 60),), 1), (((60, 20),), 1)])
def test_widest_rows_and_radius(dtype, lens, kv):
    """Heads of 128 and a radius of 1024: the most LDS that each form of the tiled kernels takes."""
    check(dtype=dtype, lens=lens, heads=2, kv_heads=kv, dim=128, radius=1024, p=0.1, seed=507)

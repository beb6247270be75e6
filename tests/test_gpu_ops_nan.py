"""A query that is not a number: its own result is none either, whether the keys are cut into slices or not, and the
other rows' are as without it, but for the last bits: rows of a wave move their running maximum
together."""
import pytest

from tests.gpu_util import announce, torch_cuda

pytestmark = pytest.mark.gpu
A = pytest.importorskip("paper_2504_13850_amd.api")


@pytest.mark.parametrize("queries,keys", [(1, 100), (1, 5000), (40, 60), (40, 3000)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_nan_query(dtype, queries, keys):
    torch = torch_cuda()
    announce(f"attention with a NaN query {dtype} {queries} {keys}")
    g = torch.Generator(device="cuda").manual_seed(1)
    make = lambda *s: torch.randn(s, generator=g, device="cuda").to(getattr(torch, dtype))  # noqa: E731
    q, k, v = make(queries, 4, 64), make(keys, 2, 64), make(keys, 2, 64)
    zero, nq, nk = (torch.tensor([n], dtype=torch.int32, device="cuda") for n in (0, queries, keys))

    def run():
        out = torch.empty_like(q)
        a = A.make_attn(q, k, v, out, zero, nq, zero, nk, queries, keys)
        ws = torch.empty(A.fo_attn_workspace(a), dtype=torch.uint8, device="cuda")
        A.fo_attn_fwd(a, q, k, v, out, None, ws)
        torch.cuda.synchronize()
        return out

    want = run()
    q[queries - 1, 1] = float("nan")
    got = run()
    assert torch.isnan(got[queries - 1, 1]).all()
    want[queries - 1, 1] = got[queries - 1, 1] = 0
    eps = {"bfloat16": 2.0 ** -7, "float32": 2.0 ** -18}[dtype]  # two roundings of a result; sums in another order
    assert float((got - want).abs().max()) <= eps * float(want.abs().max())

"""A language model's operators on rows that lie more than 2^31 elements apart."""
import numpy as np
import pytest

from tests import lm_ref as R
from tests.gpu_util import announce, torch_cuda

pytestmark = pytest.mark.gpu
A = pytest.importorskip("paper_2504_13850_amd.api")
LD, ROWS = (1 << 30) + 16, 4  # the last row starts past 2^31 elements


def _far(raw, at, cols, values=None):
    """A [ROWS, cols] matrix in raw, its rows LD apart."""
    t = raw.as_strided((ROWS, cols), (LD, 1), at)
    if values is not None:
        t.copy_(values)
    return t


def _np(t):
    return t.detach().double().cpu().numpy()


def test_rows_far_apart():
    """bf16 rows: results within 2^-8 of their value, and what 2^-20 of the terms' sizes adds (sums of up to 200 terms)."""
    torch = torch_cuda()
    announce("rows far apart")
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of GPU memory")
    raw = torch.empty(3 * LD + (1 << 16), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    near = lambda got, want, size=0.0: np.testing.assert_array_less(  # noqa: E731
        abs(_np(got) - want), 2 ** -8 * (1 + 2 ** -8) * abs(want) + 2 ** -20 * (abs(want) + size) + 1e-30)
    C = 200
    at = iter(range(0, 1 << 16, 512))
    # embedding: far tables, results and gradients
    table, tok = _far(raw, next(at), C, normal(ROWS, C)), np.array([3, -1, 0, 3], np.int32)
    tokens = torch.from_numpy(tok).cuda()
    out, dout, dtable = _far(raw, next(at), C), _far(raw, next(at), C, normal(ROWS, C)), _far(raw, next(at), C)
    A.fo_embed_fwd(tokens, table, out, scale=2.0)
    near(out, R.embed(tok, _np(table), 2.0))
    ws = torch.empty(max(A.fo_embed_workspace(ROWS, C, ROWS), A.fo_rmsnorm_workspace(ROWS, C)), dtype=torch.uint8, device="cuda")
    A.fo_embed_bwd(tokens, dout, dtable, scale=2.0, workspace=ws)
    want, size, _ = R.embed_grad(tok, _np(dout), 2.0, ROWS)
    near(dtable, want, size)
    # norm
    x, res, dy, dres = (_far(raw, next(at), C, normal(ROWS, C)) for _ in range(4))
    h, y, dx, w, dw, rstd = _far(raw, next(at), C), _far(raw, next(at), C), _far(raw, next(at), C), normal(C), normal(C), torch.empty(ROWS, device="cuda")
    A.fo_rmsnorm_fwd(x, w, y, rstd, 1e-6, residual=res, h=h)
    hh, _, yy = R.rmsnorm(_np(x), _np(res), _np(w), 1e-6)
    near(h, hh)
    near(y, yy)
    A.fo_rmsnorm_bwd(dy, h, w, rstd, dx, dw=dw, dres=dres, workspace=ws)
    wx, ww, size, sizew = R.rmsnorm_grad(_np(dy), _np(h), _np(w), _np(rstd), _np(dres))
    near(dx, wx, size)
    near(dw, ww, sizew)
    # log probabilities
    logits, d, e = _far(raw, next(at), C, normal(ROWS, C)), _far(raw, next(at), C), _far(raw, next(at), C)
    t, weight = np.array([199, 0, 7, 100], np.int32), torch.full((ROWS,), 0.25, device="cuda")
    targets, (logp, lse, loss) = torch.from_numpy(t).cuda(), torch.empty((3, ROWS), device="cuda")
    A.fo_logp_fwd(logits, targets, logp, lse)
    A.fo_logp_bwd(logits, targets, logp, lse, -weight, d)
    A.fo_xent(logits, targets, weight, loss, e)
    near(logp, R.logp(_np(logits), t, 1.0)[0])
    assert torch.equal(loss, -logp) or float((loss + logp).abs().max()) < 1e-5
    want = R.logp_grad(_np(logits), t, 1.0, -np.full(ROWS, 0.25))
    near(d, want)
    near(e, want)
    # 8-bit rows and their product, and its far result
    raw8 = torch.empty(3 * LD + (1 << 16), dtype=torch.uint8, device="cuda")
    q8, s8 = raw8.as_strided((ROWS, C), (LD, 1), 0), torch.empty(ROWS, device="cuda")
    A.fo_quant_f8(x, q8, s8)
    v = R.f8_values()[q8.cpu().numpy()]
    c = _far(raw, next(at), ROWS)
    A.fo_gemm_f8(q8, s8, q8, None, c)
    want, size = R.gemm(v, _np(s8), v, None)
    np.testing.assert_array_less(abs(_np(c) - want), 2 ** -8 * (1 + 2 ** -8) * abs(want) + 2 ** -10 * size + 1e-30)
    v = v * _np(s8)[:, None]
    np.testing.assert_array_less(abs(v - _np(x)), 2 ** -4 * abs(_np(x)) + 2 ** -9 * _np(s8)[:, None])


def test_long_table():
    """Tokens whose rows lie past 2^31 elements of a contiguous table, and its gradient's zeros there."""
    torch = torch_cuda()
    announce("long table")
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of GPU memory")
    vocab, cols = 1100003, 2000
    table = torch.empty((vocab, cols), dtype=torch.bfloat16, device="cuda")
    rows = [0, 5, vocab - 1, vocab // 2, vocab - 1]
    for r in rows:
        table[r] = r % 251
    tokens, out = torch.tensor(rows, dtype=torch.int32, device="cuda"), torch.empty((5, cols), dtype=torch.bfloat16, device="cuda")
    A.fo_embed_fwd(tokens, table, out)
    assert out[:, 7].tolist() == [float(r % 251) for r in rows]
    table.fill_(float("nan"))
    ws = torch.empty(A.fo_embed_workspace(5, cols, vocab), dtype=torch.uint8, device="cuda")
    dout = torch.arange(1.0, 6.0, device="cuda").bfloat16()[:, None].expand(5, cols).contiguous()
    A.fo_embed_bwd(tokens, dout, table, workspace=ws)
    assert float(table[0].sum()) == cols and float(table[vocab - 1, -1]) == 8 and float(table[vocab // 2, 0]) == 4
    assert int((table != 0).any(1).sum()) == 4 and not bool(table.isnan().any())

"""GPU tests of a language model's operators at the sizes that choose each of their kernels, against 64-bit torch on the
same (rounded) inputs: operands past the caches, long tiles, many rows, rows in place.  HALF: a result's rounding; F =
2^-24: an fp32 operation; a sum of n terms is off by at most n F times their sizes."""
import numpy as np
import pytest

from tests import lm_ref as R
from tests.gpu_util import announce, torch_cuda
from tests.test_gpu_lm_ops import A, F, HALF, NAN, Mat, _bytes, _dt, _norm_slack, _normal, _ws

pytestmark = pytest.mark.gpu


def _close(name, got, want, bound):
    off = ~((got.double() - want).abs() <= bound + 1e-37)
    assert not bool(off.any()), f"{name}: {int(off.sum())} values off, first at {off.nonzero()[0].tolist()}"


# ------------------------------------------------------------------ RMS norm
@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 9000, 4096), ("f32", 4500, 4096), ("bf16", 4200, 8191),
                                             ("f32", 2100, 8190), ("bf16", 2100, 16380), ("f32", 1100, 16380),
                                             ("bf16", 3400, 10007), ("bf16", 560000, 61), ("f32", 40000, 500),
                                             ("bf16", 45000, 769), ("bf16", 2001, 20003), ("f32", 1001, 33003)])
def test_norm_past_the_caches(dtype, rows, cols):
    """More than 256 MB of operands."""
    torch = torch_cuda()
    announce(f"norm past the caches, {dtype} {rows} x {cols}")
    assert 4 * rows * cols * (2 if dtype == "bf16" else 4) > 256 << 20
    dt = _dt(dtype)
    x, res, dy, dres = (_normal(s, rows, cols).to(dt) for s in (1, 2, 3, 4))
    w = (1 + 0.3 * _normal(5, cols)).to(dt)
    h, y, dx, dw, rstd = (torch.full_like(t, NAN) for t in (x, x, x, w, _normal(6, rows)))
    A.fo_rmsnorm_fwd(x, w, y, rstd, 1e-5, residual=res, h=h)
    A.fo_rmsnorm_bwd(dy, h, w, rstd, dx, dw=dw, dres=dres, workspace=_ws(A.fo_rmsnorm_workspace(rows, cols)))
    half, slack, wd = HALF[dtype] * (1 + 2 ** -8), _norm_slack(cols), w.double()
    sums, sizes = torch.zeros((2, cols), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 24) // cols)
    for r0 in range(0, rows, step):
        at = slice(r0, min(rows, r0 + step))
        hh = x[at].double() + res[at].double()
        rr = 1 / (hh.square().mean(1) + float(np.float32(1e-5))).sqrt()
        _close("h", h[at], hh, (half + F) * hh.abs())
        _close("rstd", rstd[at], rr, slack * rr)
        want = hh * rr[:, None] * wd
        _close("y", y[at], want, (half + slack) * want.abs())
        hs, r, d = h[at].double(), rstd[at].double()[:, None], dy[at].double()
        g = d * wd
        want = dres[at].double() + r * (g - hs * r * r * (g * hs).sum(1, keepdim=True) / cols)
        size = dres[at].double().abs() + r * (g.abs() + hs.abs() * r * r * (g * hs).abs().sum(1, keepdim=True) / cols)
        _close("dx", dx[at], want, half * want.abs() + slack * size)
        term = d * hs * r
        sums += term.sum(0)
        sizes += term.abs().sum(0)
    # a column's sum is cut into parts and teams: no chain of additions is as long as the rows
    _close("dw", dw, sums, half * sums.abs() + (rows / 64 + 1100) * F * sizes)


RAGGED = [101, 513, 769, 1537, 2051, 2561, 5001, 6149, 6657, 9001, 16381, 40001]  # 513 and such: the last eight begin a wave


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", RAGGED)
def test_norm_in_place_of_odd_rows(cols, dtype):
    """Results over operands have the bits of results beside them."""
    torch = torch_cuda()
    for rows in (5, 530):
        announce(f"norm in place, {dtype} {rows} x {cols}")
        dt = _dt(dtype)
        x, r, w = _normal(1, rows, cols).to(dt), _normal(2, rows, cols).to(dt), _normal(3, cols).to(dt)
        y, h, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
        A.fo_rmsnorm_fwd(x, w, y, rstd, 1e-6, residual=r, h=h)
        x2, r2 = x.clone(), r.clone()
        A.fo_rmsnorm_fwd(x2, w, x2, None, 1e-6, residual=r2, h=r2)
        assert torch.equal(x2, y) and torch.equal(r2, h)
        x2, r2 = x.clone(), r.clone()
        A.fo_rmsnorm_fwd(x2, w, r2, None, 1e-6, residual=r2, h=x2)
        assert torch.equal(r2, y) and torch.equal(x2, h)
        q, s = torch.empty((2, rows, cols), dtype=torch.uint8, device="cuda"), torch.empty((2, rows), device="cuda")
        A.fo_rmsnorm_f8(x, w, q[0], s[0], 1e-6, residual=r, h=torch.empty_like(x))
        x2 = x.clone()
        A.fo_rmsnorm_f8(x2, w, q[1], s[1], 1e-6, residual=r, h=x2)
        assert torch.equal(q[0], q[1]) and torch.equal(s[0], s[1]) and torch.equal(x2, h)
        dy, dres, dx, dw = _normal(4, rows, cols).to(dt), _normal(5, rows, cols).to(dt), torch.empty_like(x), torch.empty_like(w)
        ws = _ws(A.fo_rmsnorm_workspace(rows, cols))
        A.fo_rmsnorm_bwd(dy, h, w, rstd, dx, dw=dw, dres=dres, workspace=ws)
        for over in range(3):
            v, dw2 = [dy.clone(), dres.clone(), h.clone()], torch.empty_like(w)
            A.fo_rmsnorm_bwd(v[0], v[2], w, rstd, v[over], dw=dw2, dres=v[1], workspace=ws)
            assert torch.equal(v[over], dx)
            # few rows whose gradient lies over what dw is read from join dw in another order
            size = (dy.double() * h.double() * rstd.double()[:, None]).abs().sum(0)
            _close("dw", dw2, dw.double(), 2 * (HALF[dtype] * (1 + 2 ** -8) * dw.double().abs() + (rows + 4) * F * size))


# ------------------------------------------------------------------ log probabilities
@pytest.mark.parametrize("dtype,rows,vocab", [
    ("bf16", 3000, 32000), ("f32", 1200, 32001), ("bf16", 600000, 120), ("f32", 300001, 121), ("bf16", 70000, 1000),
    ("bf16", 40001, 2003), ("f32", 60000, 600), ("bf16", 9000, 9001), ("bf16", 1500, 50001), ("bf16", 1100, 65535),
    ("bf16", 1030, 70001),  # past the caches
    ("bf16", 5, 40000), ("f32", 3, 40007), ("bf16", 4, 60001), ("f32", 2, 65536), ("f32", 3, 65529)])
def test_logp_of_many_logits(dtype, rows, vocab):
    """A spread of 2.5 and sure targets, and some rows without one.  c: what a row's sum may be off by; the exponents'
    rounding takes 4 F of themselves (up to 45 here) and of lse (below 40)."""
    torch = torch_cuda()
    announce(f"logp, {dtype} {rows} x {vocab}")
    dt, g0 = _dt(dtype), torch.Generator(device="cuda").manual_seed(rows)
    x = _normal(1, rows, vocab, scale=2.5).to(dt)
    t = torch.randint(0, vocab, (rows,), generator=g0, device="cuda")
    row = torch.arange(rows, device="cuda")
    x[row, t] += torch.where(row % 3 == 0, 22.0, 0.0).to(dt)
    t[1::7] = -1
    targets, g = t.to(torch.int32), _normal(5, rows)
    ws = _ws(A.fo_logp_workspace(rows, vocab))
    logp, lse, loss = torch.full((3, rows), NAN, device="cuda")
    A.fo_logp_fwd(x, targets, logp, lse, scale=0.75, workspace=ws)
    d, e = torch.full_like(x, NAN), torch.full_like(x, NAN)
    A.fo_logp_bwd(x, targets, logp, lse, g, d, scale=0.75)
    A.fo_xent(x, targets, -g, loss, e, scale=0.75, workspace=ws)
    c = (64 + vocab / 1024 + 3 * 45 + 4 * 85 + 16) * F
    step = max(1, (1 << 23) // vocab)
    for r0 in range(0, rows, step):
        at = slice(r0, min(rows, r0 + step))
        z, tt = x[at].double() * 0.75, t[at]
        there, own = tt >= 0, tt.clamp_min(0)[:, None]
        z -= z.amax(1, keepdim=True)
        rest = z.exp().scatter(1, own, 0.0).sum(1)
        zt = z.gather(1, own)[:, 0]
        total = rest + zt.exp()
        lp = torch.where(zt == 0, -torch.log1p(rest), zt - total.log())
        p = z.exp() / total[:, None]
        want = (-p).scatter(1, own, (rest / total)[:, None]) * (0.75 * g[at].double())[:, None]
        want, lp = torch.where(there[:, None], want, 0.0), torch.where(there, lp, 0.0)
        off = c * (rest / total + lp.abs())
        _close("logp", logp[at], lp, off + F * lp.abs())
        _close("loss", loss[at], -lp, off + F * lp.abs())
        bound = want.abs() * (HALF[dtype] * (1 + 2 ** -8) + c)
        bound.scatter_add_(1, own, (off * g[at].abs())[:, None])
        _close("dlogits", d[at], want, bound)
        _close("dlogits of the loss", e[at], want, bound)
    over = x.clone()
    A.fo_xent(over, targets, -g, loss, over, scale=0.75, workspace=ws)
    assert torch.equal(over, e)
    A.fo_logp_bwd(x, targets, logp, lse, g, x, scale=0.75)
    assert torch.equal(x, d)


# ------------------------------------------------------------------ embedding
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,vocab", [((1 << 20) + 5, 8, 1000), ((1 << 20) + 4097, 5, 70001), (1500000, 16, 1 << 21),
                                             (1 << 20, 8, 300)])
def test_embed_gradient_of_many_rows(dtype, rows, cols, vocab):
    torch = torch_cuda()
    announce(f"embedding gradient, {dtype} {rows} rows of {cols}, vocab {vocab}")
    g = torch.Generator(device="cuda").manual_seed(rows)
    tokens = torch.randint(-1, vocab + 1, (rows,), generator=g, device="cuda")
    tokens = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.2, tokens % 3, tokens)
    dout, dtable = _normal(1, rows, cols).to(_dt(dtype)), torch.full((vocab, cols), NAN, dtype=_dt(dtype), device="cuda")
    A.fo_embed_bwd(tokens.to(torch.int32), dout, dtable, scale=0.5, workspace=_ws(A.fo_embed_workspace(rows, cols, vocab)))
    inside = (tokens >= 0) & (tokens < vocab)
    at, terms = tokens[inside], 0.5 * dout[inside].double()
    zero = torch.zeros((vocab, cols), dtype=torch.float64, device="cuda")
    want, size = zero.index_add(0, at, terms), zero.index_add(0, at, terms.abs())
    # pieces of 64 rows, an eighth of a token's pieces a team, eight teams
    chain = 64 + torch.bincount(at, minlength=vocab)[:, None] / 512 + 10
    _close("dtable", dtable, want, HALF[dtype] * want.abs() * (1 + 2 ** -8) + chain * F * size)


# ------------------------------------------------------------------ 8-bit product
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(3, 20000, 512), (16, 16390, 500), (1, 40001, 1104),     # few rows, many columns
                                   (3400, 3500, 1200), (3329, 3841, 2063),                  # 256 x 256, many steps
                                   (700, 4100, 1200), (641, 4001, 2064),                    # 128 x 128, three stages
                                   (2049, 2600, 1200), (1500, 4001, 2047),                  # 128 x 128, two stages
                                   (512, 2050, 2064), (385, 1000, 4112), (70, 300, 20016)])  # 64 x 64; slices of k
def test_gemm_f8_of_many_steps(dtype, M, N, K):
    """The stages of LDS are filled again and again.  In bf16 products are cut below 2^-13 of the largest of eight."""
    torch = torch_cuda()
    announce(f"8-bit product, {dtype} {M} x {N} x {K}")
    a, b = (torch.from_numpy(_bytes(s, n, K)).cuda() for s, n in ((M, M), (N, N)))
    sa, sb = _normal(1, M).abs() + 0.1, _normal(2, N)
    c = Mat(M, N, dtype, 3, 1)
    A.fo_gemm_f8(a, sa, b, sb, c.t, workspace=_ws(A.fo_gemm_f8_workspace(M, N, K)))
    v = torch.from_numpy(R.f8_values()).cuda()
    x, y = v[a.long()] * sa.double()[:, None], v[b.long()] * sb.double()[:, None]
    want, size = x @ y.t().contiguous(), x.abs() @ y.abs().t().contiguous()
    cut = 2.0 ** -10 if dtype == "bf16" else 0.0
    _close("c", c.t, want, HALF[dtype] * want.abs() * (1 + 2 ** -8) + ((K + 4) * F + cut) * size)
    assert c.untouched()

"""GPU tests of a language model's operators at infinite and far values, against their plain 64-bit statements
(tests/lm_ref.py).  F = 2^-24 bounds an fp32 operation, HALF a result's rounding to its type."""
import numpy as np
import pytest

from tests import lm_ref as R
from tests.gpu_util import announce, torch_cuda
from tests.test_gpu_lm_ops import A, F, HALF, NAN, _near, _normal, _np, _ws

pytestmark = pytest.mark.gpu
INF = float("inf")


def _i32(x):
    torch = torch_cuda()
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ preference loss
@pytest.mark.parametrize("smooth", [0.0, 0.1, 1.0])
def test_pref_infinite_rewards(smooth):
    """A token of probability 0 makes a reward infinite: the loss is its limit there, 0 where the term that grows has no
    weight, and the gradient stays finite.  Two rewards of the same infinity give NaN.  Other pairs do not notice.
    Gradients: three fp32 roundings."""
    torch = torch_cuda()
    announce(f"preference loss, infinite rewards, smooth {smooth}")
    spans = [(5 * q, 5 * q + 5) for q in range(10)]
    logp, ref = -_normal(1, 50).abs(), -_normal(2, 50).abs()
    logp[7] = -INF                # the rejected answer of pair 0
    logp[11] = -INF               # the chosen one of pair 1
    logp[24], logp[25] = -INF, -INF   # both of pair 2
    ref[40] = -INF                # the frozen model's, in the chosen answer of pair 4
    loss, reward, d = torch.empty(5, device="cuda"), torch.empty(10, device="cuda"), torch.empty(50, device="cuda")
    A.fo_pref_loss(logp, ref, _i32([s[0] for s in spans]), _i32([s[1] for s in spans]), loss, reward, d, beta=0.5,
                   smooth=smooth, dloss=0.25)
    sm = float(np.float32(smooth))
    limit = lambda weight: INF if weight > 0 else 0.0  # noqa: E731
    assert reward[[1, 2, 4, 5]].tolist() == [-INF] * 4 and reward[8] == INF
    assert float(loss[0]) == limit(sm) and float(loss[1]) == limit(1 - sm) and float(loss[4]) == limit(sm)
    assert loss[2].isnan() and d[20:30].isnan().all()
    want = np.repeat([sm, -sm, -(1 - sm), 1 - sm, NAN, NAN, 0, 0, sm, -sm], 5) * 0.25 * 0.5
    fine = _np(logp)[30:40], _np(ref)[30:40]
    wl, _, wd, _, dd = R.pref(*fine, [(0, 5), (5, 10)], 0.5, sm, False, 0.25)
    want[30:40] = wd
    _near("loss", _np(loss[3:4]), wl, (12 + 2 * abs(dd)) * F * wl)
    bound = 3 * F * abs(want)
    bound[30:40] = (12 + 2 * abs(dd)) * F * 0.125
    _near("dlogp", _np(d), want, np.nan_to_num(bound))


@pytest.mark.parametrize("n,apart,beta,smooth,mean", [(1500, 0.04, 0.5, 0.0, False), (1500, -0.04, 0.5, 0.0, False),
                                                      (900, 0.03, 0.5, 0.1, False), (2000, 0.3, 40.0, 0.0, True),
                                                      (37, 0.2, 0.1, 0.5, False)])
def test_pref_of_long_answers_keeps_its_bits(n, apart, beta, smooth, mean):
    """Sums and functions in 64 bits, results rounded once.  The sums are off by at most n 2^-53 of their terms' sizes,
    and loss and gradient by that, relative, for neither's logarithm is steeper than 1 in d."""
    torch = torch_cuda()
    announce(f"preference loss, answers of {n}")
    for seed in range(4):
        spans = [(0, n), (n, 2 * n + 3)]
        logp, ref = -_normal(seed, 2 * n + 3).abs() * 2, -_normal(seed + 9, 2 * n + 3).abs() * 2
        logp[:n] += apart + ref[:n] - logp[:n] + 0.01 * logp[:n]
        logp[n:] += -apart + ref[n:] - logp[n:] + 0.01 * logp[n:]
        loss, reward, d = torch.empty(1, device="cuda"), torch.empty(2, device="cuda"), torch.empty(2 * n + 3, device="cuda")
        A.fo_pref_loss(logp, ref, _i32([0, n]), _i32([n, 2 * n + 3]), loss, reward, d, beta=beta, smooth=smooth, mean=mean,
                       dloss=0.7)
        b, sm = float(np.float32(beta)), float(np.float32(smooth))
        wl, wr, wd, size, _ = R.pref(_np(logp), _np(ref), spans, b, sm, mean, float(np.float32(0.7)))
        each = b / n if mean else b
        off = 2 * (2 * n * 2.0 ** -53 * each * (abs(_np(logp)) + abs(_np(ref))).sum() + 2.0 ** -46)
        assert off < F / 8
        _near("reward", _np(reward), wr, (1 + 2 ** -8) * F * abs(wr) + off)
        _near("loss", _np(loss), wl, (1 + 2 ** -8) * F * wl + off * wl)
        _near("dlogp", _np(d), wd, (1 + 2 ** -8) * F * abs(wd) + off * size)


# ------------------------------------------------------------------ log probabilities
@pytest.mark.parametrize("rows,vocab,shift", [(50, 100, 3e4), (40, 700, -1e5), (20, 1024, 3e4), (12, 3000, 1e5),
                                              (6, 20000, -1e5), (3, 50000, 1e5), (4, 70001, 1e5), (6, 3, -3e4)])
def test_logp_gradient_of_far_logits(rows, vocab, shift):
    """Logits far from 0: the gradient is as exact as near 0.  lse is rounded to fp32, by up to |lse| F, and logp keeps
    what that loses.  A term p's exponent x = z - lse is off by F of itself for each of four operations, logp by its own
    bound (the forward tests': c and 4 F of its parts) and by F of itself on its way; the rest are some 24 operations."""
    torch = torch_cuda()
    announce(f"gradient of far logits, {rows} x {vocab}, around {shift}")
    x = _normal(rows, rows, vocab, scale=2.5)
    t = np.random.default_rng(vocab).integers(0, vocab, rows)
    at = torch.arange(rows), torch.from_numpy(t)
    x[at] += torch.tensor([0.0, 6.0, 15.0], device="cuda").repeat(rows)[:rows]
    x += shift
    targets, g = _i32(t.tolist()), _normal(5, rows)
    logp, lse = torch.full((2, rows), NAN, device="cuda")
    ws = _ws(A.fo_logp_workspace(rows, vocab))
    for scale in (1.0, 0.8):
        A.fo_logp_fwd(x, targets, logp, lse, scale=scale, workspace=ws)
        sc, z = float(np.float32(scale)), _np(x)
        lp, ls, p, miss, _, _ = R.logp(z, t, sc)
        d = torch.full_like(x, NAN)
        A.fo_logp_bwd(x, targets, logp, lse, g, d, scale=scale)
        want = R.logp_grad(z, t, sc, _np(g))
        spread = sc * (z.max(1) - z.min(1))
        c = (64 + vocab / 1024 + 3 * spread) * F
        gap = sc * (z.max(1) - z[np.arange(rows), t])
        own_off = c * miss + 4 * F * (abs(lp) + (gap > 0) * (gap + np.log(vocab) + 1))
        far = abs(sc * z - ls[:, None])
        bound = abs(want) * ((1 + 24) * F + 4 * F * far + (own_off + 2 * F * abs(lp))[:, None])
        bound[np.arange(rows), t] += abs(sc * _np(g)) * own_off
        _near("dlogits", _np(d), want, bound)
        e, loss = torch.full_like(x, NAN), torch.empty(rows, device="cuda")
        A.fo_xent(x, targets, -g, loss, e, scale=scale, workspace=ws)
        _near("dlogits of the loss", _np(e), want, bound)
        over = x.clone()
        A.fo_logp_bwd(over, targets, logp, lse, g, over, scale=scale)
        assert torch.equal(over, d)
        over = x.clone()
        A.fo_xent(over, targets, -g, loss, over, scale=scale, workspace=ws)
        assert torch.equal(over, e)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_logp_gradient_of_extreme_logits(dtype, scale):
    """Rows of nothing but a type's lowest value or another far one are uniform; a logit far above the others takes all;
    one past fp32 with its scale as well.  A uniform row's terms: exp(logp), off by 2 |logp| F and a few operations."""
    torch = torch_cuda()
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    for vocab in (5, 40, 700, 30000, 70001):
        announce(f"gradient of extreme logits, {dtype}, {vocab} of them, scale {scale}")
        x = torch.zeros((6, vocab), dtype=dt, device="cuda")
        x[0], x[1], x[2] = torch.finfo(dt).min, -1e30, 3e9
        x[3, 3], x[4, 3], x[5, 4] = 1e10, -1e10, 3e38
        targets, g = _i32([3, 2, 0, 3, 3, 4]), torch.tensor([1.0, -2.0, 0.5, 1.0, 1.0, 3.0], device="cuda")
        logp, lse = torch.empty((2, 6), device="cuda")
        ws = _ws(A.fo_logp_workspace(6, vocab))
        A.fo_logp_fwd(x, targets, logp, lse, scale=scale, workspace=ws)
        want = np.zeros((6, vocab))
        for r in range(3):
            want[r] = -1.0 / vocab
            want[r, targets[r].item()] += 1
        want[4] = -1.0 / (vocab - 1)
        want[4, 3] = 1
        want *= float(np.float32(scale)) * _np(g)[:, None]
        d, e, loss = torch.full_like(x, NAN), torch.full_like(x, NAN), torch.empty(6, device="cuda")
        A.fo_logp_bwd(x, targets, logp, lse, g, d, scale=scale)
        bound = abs(want) * (HALF[dtype] * (1 + 2 ** -8) + (4 * np.log(vocab) + 24) * F)
        _near("dlogits", _np(d), want, bound)
        A.fo_xent(x, targets, -g, loss, e, scale=scale, workspace=ws)
        _near("dlogits of the loss", _np(e), want, bound)
    x = torch.zeros((1, 40), dtype=dt, device="cuda")
    x[0, 4] = 3e38
    A.fo_logp_fwd(x, _i32([4]), logp[:1], lse[:1], scale=4.0)
    d = torch.full_like(x, NAN)
    A.fo_logp_bwd(x, _i32([4]), logp[:1], lse[:1], g[:1], d, scale=4.0)
    assert float(logp[0]) == 0 and (d == 0).all()


# ------------------------------------------------------------------ 8-bit rows
@pytest.mark.parametrize("h,w,eps", [(1e-17, 1e-29, 0.0), (1e-3, 1e-25, 1e-6), (1e-16, 1e26, 0.0), (1e15, 1e27, 1e-6),
                                     (1e15, 1e-25, 0.0)])
@pytest.mark.parametrize("cols", [90, 5003, 33001])
def test_norm_f8_of_far_operands(cols, h, w, eps):
    """h and w whose product leaves fp32's range, or its full precision, where y does not.  Tolerances: the 8-bit rows'
    of the other tests."""
    torch = torch_cuda()
    from tests.test_gpu_lm_ops import _check_f8, _norm_slack
    for dtype in (torch.float32, torch.bfloat16):
        announce(f"8-bit norm, h {h}, w {w}, {cols} columns, {dtype}")
        x, wt = (_normal(1, 5, cols) * h).to(dtype), ((1 + 0.3 * _normal(2, cols)) * w).to(dtype)
        q, s = torch.empty((5, cols), dtype=torch.uint8, device="cuda"), torch.empty(5, device="cuda")
        A.fo_rmsnorm_f8(x, wt, q, s, eps)
        y = R.rmsnorm(_np(x), None, _np(wt), float(np.float32(eps)))[2]
        assert (abs(y).max(1) > 2.0 ** -100).all()
        _check_f8(y, q.cpu().numpy(), _np(s), _norm_slack(cols))


# ------------------------------------------------------------------ 8-bit product
def test_gemm_f8_without_a_workspace():
    """As its workspace call says: few rows, long k and odd k among them, and a small product of odd rows."""
    torch = torch_cuda()
    for M, N, K in ((4, 4096, 8192), (16, 64, 65536), (32, 512, 16400), (7, 100, 9001), (40, 100, 9001)):
        announce(f"8-bit product without a workspace, {M} x {N} x {K}")
        assert A.fo_gemm_f8_workspace(M, N, K) == 0
        v = R.f8_values()
        a, b = (np.random.default_rng(n).integers(0, 0x7F, (n, K)).astype(np.uint8) for n in (M, N))
        c = torch.empty((M, N), device="cuda")
        A.fo_gemm_f8(torch.from_numpy(a).cuda(), None, torch.from_numpy(b).cuda(), None, c)
        want, size = R.gemm(v[a], None, v[b], None)
        _near("c", _np(c), want, HALF["f32"] * abs(want) + (K + 4) * F * size)

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

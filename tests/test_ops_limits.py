"""CPU tests of the operators' entry points at the ends of their arguments' ranges: what the kernels could not address or
represent is refused before any launch."""
import ctypes as C

import numpy as np
import pytest

from tests.test_ops_host import _record

A = pytest.importorskip("paper_2504_13850_amd.api")
MANY = (1 << 31) - 1  # the most rows there may be


def _refused(a):
    x = np.zeros(64, np.int64).ctypes.data
    return (A.lib().fo_attn_workspace(C.byref(a), 1) == -1
            and A.lib().fo_attn_fwd(C.byref(a), x, x, x, x, None, x, 1 << 62, None) == A.FO_EINVAL
            and A.lib().fo_attn_bwd(C.byref(a), x, x, x, x, x, x, x, x, x, None, x, 1 << 62, None) == A.FO_EINVAL)


@pytest.mark.parametrize("bad", [dict(q_rows=MANY, q_ld=1 << 40), dict(q_rows=MANY, out_ld=1 << 40),
                                 dict(k_rows=MANY, k_ld=1 << 40), dict(k_rows=MANY, v_ld=1 << 32),
                                 dict(q_rows=MANY, q_ld=1 << 31, dtype=1, q_hs=64)],
                         ids=lambda b: ",".join(f"{k}={v}" for k, v in b.items()))
def test_attention_offsets_past_64_bits(bad):
    """bf16 (dtype 0) elements take two bytes, fp32 four: the last one's offset has to stay below 2^63 bytes."""
    assert _refused(_record(**bad))


def test_attention_offsets_within_64_bits():
    a = _record(q_rows=MANY, q_ld=1 << 31)
    assert A.lib().fo_attn_workspace(C.byref(a), 0) >= 0


def test_dropout_offsets_past_64_bits():
    L, x = A.lib(), np.zeros(64, np.int64).ctypes.data
    far = 1 << 31
    for xl, rl, yl in ((far, 8, 8), (8, far, 8), (8, 8, far)):
        assert L.fo_dropout_fwd(A.FO_DT_F32, MANY, 8, x, xl, None, x, rl, 0.1, 1, 1, x + 64, yl, None) == A.FO_EINVAL
    for xl, yl in ((far, 8), (8, far)):
        assert L.fo_dropout_bwd(A.FO_DT_F32, MANY, 8, x, xl, 0.1, 1, 1, x + 64, yl, None, None, 0, None) == A.FO_EINVAL


@pytest.mark.parametrize("bad", [dict(cap=3e38), dict(cap=1e-40), dict(scale=3e38), dict(scale=-3e38),
                                 dict(scale=1e30, cap=1e-10)],
                         ids=lambda b: ",".join(f"{k}={v}" for k, v in b.items()))
def test_factors_past_fp32(bad):
    """scale log2(e), cap log2(e) and scale / cap are the kernels' factors; an infinite one makes every score NaN."""
    assert _refused(_record(**bad))


def test_factors_within_fp32():
    for good in (dict(cap=1e38), dict(cap=1e-37), dict(scale=2e38), dict(scale=0.0), dict(scale=0.0, cap=1e-40)):
        a = _record(**good)
        assert A.lib().fo_attn_workspace(C.byref(a), 1) >= 0, good


def test_dropout_in_place_with_another_stride():
    """Rows written over others that are still to be read."""
    L, x = A.lib(), np.zeros(64, np.int64).ctypes.data
    fwd = lambda xl, r, rl, y, yl: L.fo_dropout_fwd(  # noqa: E731
        A.FO_DT_BF16, 3, 8, x, xl, None, r, rl, 0.1, 1, 1, y, yl, None)
    assert fwd(16, None, 0, x, 8) == A.FO_EINVAL and fwd(8, None, 0, x, 16) == A.FO_EINVAL
    assert fwd(8, x + 256, 16, x + 256, 8) == A.FO_EINVAL
    for xl, yl in ((16, 8), (8, 16)):
        assert L.fo_dropout_bwd(A.FO_DT_BF16, 3, 8, x, xl, 0.1, 1, 1, x, yl, None, None, 0, None) == A.FO_EINVAL

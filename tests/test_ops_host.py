"""CPU tests of the transformer operators: the generator's known answers, the
distance buckets, the reference's gradients against differences, and what the
entry points refuse (before any launch, so no GPU is touched)."""
import ctypes as C
import math

import numpy as np
import pytest

from tests import ops_ref as R

A = pytest.importorskip("paper_2504_13850_amd.api")


def test_generator_known_answers():
    """The published answers of Philox 4x32 with seven rounds: zeros, ones, digits of pi."""
    for ctr, key, want in (
            ((0,) * 4, 0, (0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48)),
            ((0xFFFFFFFF,) * 4, 0xFFFFFFFFFFFFFFFF, (0x5207DDC2, 0x45165E59, 0x4D8EE751, 0x8C52F662)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), 0x299F31D0A4093822,
             (0x4DFCCABA, 0x190A87F0, 0xC47362BA, 0xB6B5242A))):
        assert tuple(int(x) for x in R.philox7(*ctr, key)) == want


@pytest.mark.parametrize("n,radius,causal", [(32, 128, False), (32, 128, True), (16, 32, False), (4, 5, False),
                                             (2, 2, True), (64, 1024, False), (8, 7, True)])
def test_buckets(n, radius, causal):
    got = A.fo_relpos_buckets(n, radius, causal)
    half = n if causal else n // 2
    near = half // 2
    assert len(got) == 2 * radius + 1 and got.min() == 0 and got.max() == n - 1
    for d in range(-radius, radius + 1):
        a = max(0, -d) if causal else abs(d)
        b = got[d + radius] - (half if d > 0 and not causal else 0)
        if a < near:
            assert b == a
        else:  # a^(half - near) against near^(half - b) radius^(b - near), in whole numbers
            s = half - near
            reached = [t for t in range(s + 1) if a ** s * near ** t >= near ** s * radius ** t]
            assert b == min(half - 1, near + max(reached))
    assert (np.diff(got[: radius + 1]) <= 0).all()


@pytest.mark.parametrize("n,radius,causal", [(1, 8, True), (3, 8, False), (2, 8, False), (32, 8, False),
                                             (32, 1025, False), (2048, 1000, True), (32, -1, False)])
def test_buckets_refuse(n, radius, causal):
    with pytest.raises(A.FoError):
        A.fo_relpos_buckets(n, radius, causal)


def test_reference_gradients_against_differences():
    """Central differences of the plain statement along random directions: 64 bits, step 1e-5, so their error is about
    1e-10 of the curvature; 1e-6 is asked."""
    rng = np.random.default_rng(3)
    spans = [(0, 5, 0, 5), (5, 9, 5, 11), (9, 13, 11, 13)]
    q, k, v = (rng.standard_normal(s) for s in ((13, 4, 6), (13, 2, 6), (13, 2, 6)))
    table, dout = rng.standard_normal((4, 4)), rng.standard_normal(q.shape)
    kw = dict(mask=2, scale=0.7, cap=1.5, prefix=[2, 0, 1], bucket=np.array([0, 1, 1, 2, 3, 3, 0]), p=0.3, seed=77,
              offset=5)
    got, _ = R.attention(q, k, v, spans, table=table, dout=dout, **kw)
    f = lambda q, k, v, t: (R.attention(q, k, v, spans, table=t, **kw)[0]["out"][0] * dout).sum()  # noqa: E731
    for i, name in enumerate(("dq", "dk", "dv", "dtable")):
        x = [q, k, v, table]
        d = rng.standard_normal(x[i].shape)
        up, dn = ([y + (s * 1e-5 * d if j == i else 0) for j, y in enumerate(x)] for s in (1, -1))
        want = (f(*up) - f(*dn)) / 2e-5
        assert abs((got[name][0] * d).sum() - want) <= 1e-6 * max(1, abs(want)), name


def _record(**kw):
    """A valid record over host addresses (never launched)."""
    one = np.zeros(64, np.int32)
    a = A.fo_attn(A.FO_DT_BF16, 2, 4, 2, 64, 16, 16, 32, 32, *([one.ctypes.data] * 4), 256, 64, 128, 64, 128, 64, 256,
                  64, 0.125, 0.0, A.FO_ATTN_FULL, None, None, None, 0, 0, 0.0, 1, 1)
    a.keep = one
    for n, v in kw.items():
        setattr(a, n, one.ctypes.data if v == "ptr" else v)
    return a


BAD = [dict(dtype=2), dict(batch=0), dict(heads=0), dict(kv_heads=3), dict(kv_heads=0), dict(head_dim=0),
       dict(head_dim=129), dict(max_q=-1), dict(max_k=-1), dict(q_rows=-1), dict(k_rows=1 << 31), dict(q_begin=None),
       dict(k_end=None), dict(q_ld=255), dict(q_hs=63), dict(k_ld=-1), dict(out_ld=0), dict(v_ld=1 << 50),
       dict(scale=math.nan), dict(scale=math.inf), dict(cap=-1.0), dict(cap=math.nan), dict(mask=3), dict(mask=2),
       dict(prefix="ptr"), dict(table="ptr"), dict(bucket="ptr"), dict(table="ptr", bucket="ptr"),
       dict(table="ptr", bucket="ptr", n_buckets=4, radius=1025), dict(table="ptr", bucket="ptr", n_buckets=2000),
       dict(p=1.0), dict(p=-0.1), dict(p=math.nan), dict(batch=65535, heads=65534, max_q=1 << 20)]


@pytest.mark.parametrize("bad", BAD, ids=lambda b: ",".join(f"{k}={v}" for k, v in b.items()))
def test_attention_refuses(bad):
    a = _record(**bad)
    assert A.lib().fo_attn_workspace(C.byref(a), 1) == -1 and A.last_error()
    x = np.zeros(64, np.int64).ctypes.data
    assert A.lib().fo_attn_fwd(C.byref(a), x, x, x, x, None, x, 1 << 40, None) == A.FO_EINVAL
    assert A.lib().fo_attn_bwd(C.byref(a), x, x, x, x, x, x, x, x, x, None, x, 1 << 40, None) == A.FO_EINVAL


def test_attention_refuses_operands():
    a, L = _record(), A.lib()
    x = np.zeros(64, np.int64).ctypes.data
    assert L.fo_attn_workspace(C.byref(a), 1) > 0
    assert L.fo_attn_fwd(None, x, x, x, x, None, x, 1 << 40, None) == A.FO_EINVAL
    for i in range(4):
        args = [x] * 4
        args[i] = None
        assert L.fo_attn_fwd(C.byref(a), *args, None, x, 1 << 40, None) == A.FO_EINVAL
        args[i] = x + 1
        assert L.fo_attn_fwd(C.byref(a), *args, None, x, 1 << 40, None) == A.FO_EINVAL
    for i in range(9):  # q, k, v, out, lse, dout, dq, dk, dv
        args = [x] * 9
        args[i] = None
        assert L.fo_attn_bwd(C.byref(a), *args, None, x, 1 << 40, None) == A.FO_EINVAL
    assert L.fo_attn_bwd(C.byref(a), *([x] * 9), x, x, 1 << 40, None) == A.FO_EINVAL      # dtable without a table
    assert L.fo_attn_bwd(C.byref(a), *([x] * 9), None, x, 8, None) == A.FO_EINVAL         # workspace too small
    assert L.fo_attn_bwd(C.byref(a), *([x] * 9), None, None, 1 << 40, None) == A.FO_EINVAL
    assert L.fo_attn_bwd(C.byref(a), *([x] * 9), None, x + 4, 1 << 40, None) == A.FO_EINVAL


def test_dropout_refuses():
    L, x = A.lib(), np.zeros(64, np.int64).ctypes.data
    fwd = lambda dt=0, rows=4, cols=8, xp=x, xl=8, b=None, r=None, rl=0, p=0.1, y=x, yl=8: L.fo_dropout_fwd(  # noqa: E731
        dt, rows, cols, xp, xl, b, r, rl, p, 1, 1, y, yl, None)
    for bad in (dict(dt=2), dict(rows=-1), dict(cols=0), dict(xp=None), dict(y=None), dict(xl=7), dict(yl=7),
                dict(r=x, rl=7), dict(p=1.0), dict(p=-0.5), dict(p=math.nan), dict(xp=x + 1), dict(b=x + 1)):
        assert fwd(**bad) == A.FO_EINVAL, bad
    bwd = lambda dt=0, rows=4, cols=8, dy=x, dyl=8, p=0.1, dx=x, dxl=8, db=None, ws=x, n=1 << 30: L.fo_dropout_bwd(  # noqa: E731
        dt, rows, cols, dy, dyl, p, 1, 1, dx, dxl, db, ws, n, None)
    for bad in (dict(dt=-1), dict(dy=None), dict(dx=None), dict(dyl=7), dict(dxl=7), dict(p=1.5),
                dict(db=x, n=0), dict(db=x, ws=None), dict(db=x, ws=x + 4), dict(db=x + 1)):
        assert bwd(**bad) == A.FO_EINVAL, bad
    assert fwd(rows=0, xp=None, y=None) == A.FO_OK
    assert L.fo_dropout_workspace(-1, 8) == -1 and L.fo_dropout_workspace(4, 0) == -1


def test_binding_refuses_other_tensors():
    import torch
    t = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    i = torch.zeros(1, dtype=torch.int32)
    ok = dict(q=t(4, 2, 8), k=t(4, 2, 8), v=t(4, 2, 8), out=t(4, 2, 8), q_begin=i, q_end=i, k_begin=i, k_end=i,
              max_q=4, max_k=4)
    A.make_attn(**ok)
    for bad in (dict(k=t(4, 2, 9)), dict(v=t(5, 2, 8)), dict(out=t(4, 1, 8)), dict(k=t(4, 2, 8, dt=torch.float32)),
                dict(q=t(4, 2, 8, dt=torch.float16)), dict(q=t(4, 2, 16)[..., ::2]), dict(q_begin=i.long()),
                dict(k_end=torch.zeros(2, dtype=torch.int32)), dict(table=t(4, 2)),
                dict(table=t(4, 3), bucket=torch.zeros(5, dtype=torch.int32)),
                dict(table=t(4, 2), bucket=torch.zeros(4, dtype=torch.int32)),
                dict(table=t(4, 2, dt=torch.float32), bucket=torch.zeros(5, dtype=torch.int32))):
        with pytest.raises(A.FoError):
            A.make_attn(**{**ok, **bad})
    with pytest.raises(A.FoError):
        A.fo_dropout_fwd(t(4, 8), t(4, 9), 0.1, 1, 1)
    with pytest.raises(A.FoError):
        A.fo_dropout_bwd(t(4, 8), t(4, 8), 0.1, 1, 1, dbias=t(7))

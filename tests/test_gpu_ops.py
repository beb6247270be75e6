"""GPU tests of the transformer operators against their plain 64-bit statements
(tests/ops_ref.py), on the kernels' own (rounded) inputs.

Error bounds.  bf16 keeps eight significant bits: a rounding is off by 2^-8 at
most and by less than 2^-9 in the root mean square.  A result is rounded once to
its type and, in bf16, is a sum of terms that were rounded once themselves, their
errors independent: less than 2^-9 of the root of the terms' summed squares,
which the statement returns beside each value.  Over a whole result both get a
factor of two: 2^-8.  In fp32 a term's error is that of exp(u - m), u a sum
over the head: some tens of 2^-24; 2^-18 is asked.
"""
import numpy as np
import pytest

from tests import ops_ref as R
from tests.gpu_util import announce, torch_cuda

pytestmark = pytest.mark.gpu
A = pytest.importorskip("paper_2504_13850_amd.api")
EPS = {"bf16": 2.0 ** -8, "f32": 2.0 ** -18}


def _dt(name):
    torch = torch_cuda()
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _np(t):
    return t.detach().double().cpu().numpy()


def _check(name, got, value, scale, eps):
    """2-norm of the error over the written elements; the others (NaN in value) have to be untouched (NaN)."""
    got = np.asarray(got, np.float64)
    there = ~np.isnan(value)
    assert np.isnan(got[~there]).all(), f"{name}: rows of no sequence were written"
    err = np.linalg.norm((got - value)[there])
    lim = eps * (np.linalg.norm(value[there]) + np.linalg.norm(scale[there])) + 1e-30
    assert err <= lim, f"{name}: error {err:.3g}, bound {lim:.3g}"
    if there.any():  # and no single element far off
        big = np.abs((got - value)[there]).max()
        top = np.abs(value[there]).max() + np.abs(scale[there]).max()
        assert big <= 8 * eps * top + 1e-30, f"{name}: largest error {big:.3g} of {top:.3g}"


class Case:
    """Operands of one attention call.  gap: rows of no sequence (filled with NaN) before each sequence; layout:
    "fused" (q, k, v columns of one matrix, where queries and keys share rows), "rows" ([rows][heads][dim]),
    "heads" ([heads][rows][dim]) or "odd" (odd row strides, unaligned starts)."""

    def __init__(self, dtype="bf16", lens=((40, 40),), heads=2, kv_heads=None, dim=64, mask=0, cap=0.0, radius=None,
                 n_buckets=8, p=0.0, prefix=None, layout="rows", gap=0, train=True, seed=0, scale=None, hide=None):
        torch = torch_cuda()
        self.dtype, self.p, self.mask, self.cap, self.train = dtype, p, mask, cap, train
        self.eps, dt = EPS[dtype], _dt(dtype)
        kv = kv_heads or heads
        g = torch.Generator(device="cuda").manual_seed(1000 + seed)
        spans, rq, rk = [], 0, 0
        for lq, lk in lens:
            spans.append((rq + gap, rq + gap + lq, rk + gap, rk + gap + lk))
            rq, rk = rq + gap + lq, rk + gap + lk
        rq, rk = rq + gap, rk + gap
        self.spans = spans

        def fill(x, lo_hi):
            x.fill_(float("nan"))
            for lo, hi in lo_hi:
                x[lo:hi] = torch.randn((hi - lo,) + tuple(x.shape[1:]), generator=g, device="cuda").to(dt)
            return x

        def make(rows, n, how=None):
            how = how or layout
            if how == "heads":
                return torch.empty((n, rows, dim), dtype=dt, device="cuda").transpose(0, 1)
            if how == "odd":
                flat = torch.empty(rows * (n * dim + 3) + 8, dtype=dt, device="cuda")
                return flat[1:1 + rows * (n * dim + 3)].view(rows, n * dim + 3)[:, :n * dim].unflatten(1, (n, dim))
            return torch.empty((rows, n, dim), dtype=dt, device="cuda")

        qs, ks = [s[:2] for s in spans], [s[2:] for s in spans]
        if layout == "fused":
            assert qs == ks

            def trio():
                m = torch.empty((rq, (heads + 2 * kv) * dim), dtype=dt, device="cuda").fill_(float("nan"))
                return [t.unflatten(1, (-1, dim)) for t in m.split((heads * dim, kv * dim, kv * dim), 1)]
        else:
            def trio():
                return [make(rq, heads), make(rk, kv), make(rk, kv)]
        self.q, self.k, self.v = (fill(t, s) for t, s in zip(trio(), (qs, ks, ks)))
        self.grads = [t.fill_(float("nan")) for t in trio()]
        self.out = make(rq, heads, "rows" if layout == "fused" else None).fill_(float("nan"))
        self.dout = fill(make(rq, heads, "rows" if layout == "fused" else None), qs)
        self.lse = torch.full((heads, rq), float("nan"), device="cuda")
        on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.bounds = [on([s[i] for s in spans]) for i in range(4)]
        self.prefix = on(prefix) if prefix is not None else None
        self.table = self.bucket = self.dtable = None
        if radius is not None:
            self.table = torch.randn((n_buckets, heads), generator=g, device="cuda").to(dt)
            if hide is not None:  # a bucket hidden by -infinity, or by the type's lowest value
                self.table[1] = -float("inf") if hide == "inf" else torch.finfo(dt).min
            rng = np.random.default_rng(seed)
            self.bucket = on(rng.integers(0, n_buckets, 2 * radius + 1).tolist())
            self.dtable = torch.full_like(self.table, float("nan"))
        self.scale = dim ** -0.5 if scale is None else scale
        self.seed, self.offset = 0x9E3779B97F4A7C15 + seed, 7 + seed
        self.max = [max([s[1] - s[0] for s in spans]), max([s[3] - s[2] for s in spans])]
        self.a = A.make_attn(self.q, self.k, self.v, self.out, *self.bounds, *self.max, scale=self.scale, cap=cap,
                             mask=mask, prefix=self.prefix, table=self.table, bucket=self.bucket, p=p, seed=self.seed,
                             offset=self.offset)
        n = A.fo_attn_workspace(self.a, train)
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN in fp32

    def run(self, stream=None):
        A.fo_attn_fwd(self.a, self.q, self.k, self.v, self.out, self.lse if self.train else None, self.ws,
                      stream=stream)
        if self.train:
            A.fo_attn_bwd(self.a, self.q, self.k, self.v, self.out, self.lse, self.dout, *self.grads, self.dtable,
                          self.ws, stream=stream)

    def outputs(self):
        return [self.out] + (self.grads + ([self.dtable] if self.dtable is not None else []) if self.train else [])

    def verify(self):
        ref, lse = R.attention(_np(self.q), _np(self.k), _np(self.v), self.spans, self.mask, self.scale, self.cap,
                               None if self.prefix is None else self.prefix.tolist(),
                               None if self.table is None else _np(self.table),
                               None if self.bucket is None else self.bucket.cpu().numpy(), self.p, self.seed,
                               self.offset, _np(self.dout) if self.train else None)
        got = dict(zip(["out", "dq", "dk", "dv", "dtable"], self.outputs()))
        for n, (value, scale) in ref.items():
            _check(n, _np(got[n]), value, scale, self.eps)
        if self.train:
            x, there = _np(self.lse) * np.log(2), ~np.isnan(lse)  # held in base 2
            assert np.isnan(x[~there]).all()
            same = np.isinf(lse) == np.isinf(x)
            assert same[there].all()
            fin = there & np.isfinite(lse)
            assert np.abs(x[fin] - lse[fin]).max(initial=0) <= 2.0 ** -16 * (1 + np.abs(lse[fin]).max(initial=0))


def check(**kw):
    announce(f"attention {kw}")
    c = Case(**kw)
    c.run()
    c.verify()


# self-attention: (dtype, lengths, heads, kv_heads, dim, mask, cap, radius, p, layout)
SELF = [
    ("bf16", (128, 32, 77, 1), 12, 12, 64, 0, 0.0, 128, 0.1, "fused"),     # the BERT block
    ("f32", (64, 4, 33), 5, 5, 20, 0, 0.0, 32, 0.2, "fused"),              # the paper's Transformer-6
    ("f32", (256, 16, 100), 50, 50, 2, 0, 30.0, None, 0.0, "fused"),       # Transformer-12
    ("bf16", (300, 129, 64), 8, 2, 128, 1, 5.0, None, 0.0, "fused"),       # grouped heads, causal, capped
    ("bf16", (257, 200), 6, 2, 64, 2, 0.0, 16, 0.0, "fused"),              # prefix with bias
    ("bf16", (1,), 1, 1, 1, 0, 0.0, None, 0.0, "rows"),
    ("f32", (1, 2, 3), 2, 1, 3, 1, 2.0, 2, 0.5, "rows"),
    ("bf16", (31, 32, 33, 63, 65), 3, 3, 32, 1, 0.0, 7, 0.25, "heads"),
    ("bf16", (127, 129), 2, 1, 77, 2, 4.0, 1024, 0.1, "odd"),
    ("f32", (127, 129), 2, 2, 77, 1, 4.0, 40, 0.1, "odd"),
    ("f32", (190, 66), 4, 1, 128, 2, 0.0, 0, 0.0, "heads"),
    ("bf16", (100, 90), 4, 4, 100, 0, 0.0, None, 0.9, "rows"),
    ("f32", (300,), 3, 3, 64, 0, 0.0, 100, 0.0, "rows"),
    ("bf16", (700, 3), 2, 2, 48, 1, 0.0, 60, 0.0, "rows"),
    ("bf16", (513,), 4, 2, 128, 0, 0.0, 300, 0.1, "fused"),
    ("f32", (513,), 2, 1, 96, 2, 3.0, 20, 0.1, "fused"),
    ("bf16", (700,), 1, 1, 16, 0, 2.0, 20, 0.0, "rows"),
]


@pytest.mark.parametrize("i", range(len(SELF)), ids=lambda i: "-".join(map(str, SELF[i])).replace(" ", ""))
def test_self_attention(i):
    dtype, lens, heads, kv, dim, mask, cap, radius, p, layout = SELF[i]
    check(dtype=dtype, lens=tuple((n, n) for n in lens), heads=heads, kv_heads=kv, dim=dim, mask=mask, cap=cap,
          radius=radius, p=p, layout=layout, prefix=[n // 3 for n in lens] if mask == 2 else None, gap=i % 3, seed=i)


# queries and keys of different lengths; causal rows before the first key see nothing
CROSS = [((5, 40), (40, 5), (1, 70)), ((64, 1), (1, 1), (130, 64)), ((33, 0), (20, 20), (0, 9)),
         ((0, 0), (7, 300)), ((200, 90),)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", [0, 1, 2])
@pytest.mark.parametrize("i", range(len(CROSS)))
def test_lengths_and_empty_rows(dtype, mask, i):
    lens = CROSS[i]
    check(dtype=dtype, lens=lens, heads=4, kv_heads=2, dim=(64, 20)[i % 2], mask=mask, cap=(0.0, 3.0)[i % 2],
          radius=(9, None)[i % 2], p=(0.0, 0.3)[i // 2 % 2], layout="rows", gap=2, seed=100 + i,
          prefix=[(lk + 1) // 2 if b % 2 else 0 for b, (_, lk) in enumerate(lens)] if mask == 2 else None)


# heads of a few columns: (dtype, lengths, heads, kv_heads, dim, mask, cap, radius, p, layout)
NARROW = [
    ("f32", (256, 16, 100, 65), 6, 6, 2, 1, 0.0, 1024, 0.1, "fused"), ("bf16", (200, 64), 4, 2, 8, 2, 3.0, 40, 0.2, "rows"),
    ("f32", (300, 33), 4, 1, 5, 0, 2.0, 0, 0.0, "odd"), ("bf16", (129, 257), 3, 3, 3, 1, 0.0, None, 0.3, "heads"),
    ("f32", (1100,), 2, 1, 1, 1, 0.0, 20, 0.0, "rows"), ("bf16", (64,), 12, 2, 2, 0, 0.0, 100, 0.0, "rows"),
    ("f32", (700, 200), 8, 2, 8, 2, 0.0, 64, 0.1, "heads")]


@pytest.mark.parametrize("i", range(len(NARROW)), ids=lambda i: "-".join(map(str, NARROW[i])).replace(" ", ""))
def test_narrow_heads(i):
    dtype, lens, heads, kv, dim, mask, cap, radius, p, layout = NARROW[i]
    check(dtype=dtype, lens=tuple((n, n) for n in lens), heads=heads, kv_heads=kv, dim=dim, mask=mask, cap=cap,
          radius=radius, p=p, layout=layout, prefix=[n // 3 for n in lens] if mask == 2 else None, gap=i % 3,
          seed=300 + i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", [0, 1, 2])
def test_narrow_lengths_and_empty_rows(dtype, mask):
    lens = ((40, 5), (5, 70), (64, 1), (1, 1), (33, 0), (0, 9), (130, 64), (60, 2000))
    check(dtype=dtype, lens=lens, heads=4, kv_heads=2, dim=4, mask=mask, cap=3.0, radius=9, p=0.3, gap=1, seed=320,
          prefix=[(lk + 1) // 2 if b % 2 else 0 for b, (_, lk) in enumerate(lens)] if mask == 2 else None)


# sequences that one workgroup holds: (dtype, lengths, heads, dim, mask, cap, radius, p)
SHORT = [("bf16", ((128, 128), (1, 128), (128, 1), (33, 97)), 3, 64, 0, 0.0, 50, 0.2),
         ("bf16", ((64, 64), (17, 3), (0, 40), (50, 0), (31, 33)), 4, 128, 1, 3.0, 64, 0.1),
         ("f32", ((128, 100), (65, 64), (10, 128)), 2, 64, 2, 2.0, 1024, 0.3),
         ("f32", ((64, 64), (1, 1), (40, 20), (2, 64)), 5, 20, 1, 0.0, 0, 0.0),
         ("bf16", ((127, 65), (96, 128)), 2, 48, 2, 0.0, None, 0.0), ("f32", ((90, 90),), 2, 100, 0, 0.0, 20, 0.1),
         ("bf16", ((100, 128), (128, 90)), 2, 80, 1, 50.0, 1024, 0.0)]


@pytest.mark.parametrize("i", range(len(SHORT)), ids=lambda i: "-".join(map(str, SHORT[i])).replace(" ", ""))
def test_short_sequences(i):
    dtype, lens, heads, dim, mask, cap, radius, p = SHORT[i]
    check(dtype=dtype, lens=lens, heads=heads, dim=dim, mask=mask, cap=cap, radius=radius, p=p, layout=("rows", "heads")[i % 2],
          gap=1 + i % 2, seed=400 + i,
          prefix=[(lk + 1) // 2 if b % 2 else 0 for b, (_, lk) in enumerate(lens)] if mask == 2 else None)


def test_negative_and_zero_scale():
    for k, scale in enumerate((-0.3, 0.0)):
        for cap in (0.0, 2.0):
            check(dtype="bf16", lens=((70, 70),), heads=2, dim=64, mask=1, cap=cap, scale=scale, radius=8, seed=330 + k)
            check(dtype="f32", lens=((70, 70),), heads=2, dim=6, mask=1, cap=cap, scale=scale, seed=340 + k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hide", ["inf", "lowest"])
def test_hidden_distances(dtype, hide):
    check(dtype=dtype, lens=((90, 90), (1, 1), (40, 130)), heads=3, dim=32, mask=1, radius=30, n_buckets=3, hide=hide,
          seed=5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Scores of some hundreds: the softmax is nearly one-hot, and sums of exponentials unshifted would overflow."""
    check(dtype=dtype, lens=((150, 150), (70, 70)), heads=2, dim=64, mask=1, scale=10.0, seed=9)


# single tokens against a cache: (dtype, key lengths, heads, kv_heads, dim, cap, radius)
ONE = [("bf16", (1, 100, 37, 0), 12, 12, 64, 0.0, 64), ("bf16", (5000, 4097, 63), 8, 2, 128, 50.0, 128),
       ("f32", (1000, 1, 640), 5, 5, 20, 3.0, None), ("f32", (2000, 129), 12, 1, 128, 0.0, 200),
       ("bf16", (9000,), 4, 1, 64, 0.0, None), ("bf16", (300, 301), 32, 1, 77, 0.0, 5), ("bf16", (70,), 80, 2, 128, 0.0, 9),
       ("f32", (5000,), 2, 2, 2, 0.0, None)]


@pytest.mark.parametrize("i", range(len(ONE)), ids=lambda i: "-".join(map(str, ONE[i])).replace(" ", ""))
def test_single_tokens(i):
    dtype, lens, heads, kv, dim, cap, radius = ONE[i]
    check(dtype=dtype, lens=tuple((1, n) for n in lens), heads=heads, kv_heads=kv, dim=dim, cap=cap, radius=radius,
          layout=("rows", "heads", "odd")[i % 3], gap=3, train=False, seed=200 + i)


@pytest.mark.parametrize("dtype,lens,heads,kv,mask", [
    ("bf16", ((3, 4000), (7, 2500)), 4, 4, 1), ("bf16", ((20, 3000),), 8, 2, 0), ("f32", ((5, 3000), (1, 70)), 4, 1, 1),
    ("bf16", ((200, 2100),), 2, 1, 1), ("f32", ((130, 1500),), 2, 1, 2)])
def test_few_queries_many_keys(dtype, lens, heads, kv, mask):
    check(dtype=dtype, lens=lens, heads=heads, kv_heads=kv, dim=64, mask=mask, radius=50, train=False, gap=1,
          prefix=[700] if mask == 2 else None, seed=31)


def test_training_against_many_keys():
    """Few queries, many keys, and the other way round: what one side's gradient sums over is long."""
    check(dtype="bf16", lens=((10, 1500),), heads=4, kv_heads=1, dim=64, radius=40, p=0.1, seed=41)
    check(dtype="f32", lens=((1500, 10),), heads=2, kv_heads=1, dim=64, radius=40, seed=42)


def test_same_bits_again_on_another_stream():
    """A second run, on a side stream, gives the same bits: no sum depends on timing."""
    torch = torch_cuda()
    kw = dict(dtype="bf16", lens=((300, 300), (90, 90)), heads=4, kv_heads=2, dim=64, mask=1, cap=5.0, radius=20, p=0.1)
    announce(f"attention twice {kw}")
    a, b = Case(**kw), Case(**kw)
    a.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.run(stream=s)
    torch.cuda.synchronize()
    for x, y in zip(a.outputs(), b.outputs()):
        assert torch.equal(x.contiguous().view(torch.int16), y.contiguous().view(torch.int16))


def test_graph_replays():
    """Captured once, replayed on new inputs with eager work in between."""
    torch = torch_cuda()
    kw = dict(dtype="bf16", lens=((120, 120), (200, 200)), heads=4, dim=64, mask=1, radius=20, p=0.1, seed=3)
    announce(f"attention graph {kw}")
    c = Case(**kw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.run(stream=s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.run(stream=s)
    for k in range(3):
        gen = torch.Generator(device="cuda").manual_seed(50 + k)
        for t in (c.q, c.k, c.v, c.dout):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda").to(t.dtype))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        c.verify()


def test_offsets_past_32_bits():
    """A cache whose last rows lie more than 2^32 elements from its first."""
    torch = torch_cuda()
    rows, ld = 5000, 1 << 20
    announce("attention over a cache of 10 GB")
    g = torch.Generator(device="cuda").manual_seed(1)
    big = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    k, v = (big.as_strided((rows, 1, 64), (ld, 64, 1), off) for off in (0, 64))
    for t in (k, v):
        t.copy_(torch.randn((rows, 1, 64), generator=g, device="cuda").to(torch.bfloat16))
    q = torch.randn((2, 4, 64), generator=g, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    on = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    bounds = [on(0, 1), on(1, 2), on(0, 3000), on(3000, 5000)]
    a = A.make_attn(q, k, v, out, *bounds, 1, 3000)
    ws = torch.empty(A.fo_attn_workspace(a), dtype=torch.uint8, device="cuda")
    A.fo_attn_fwd(a, q, k, v, out, None, ws)
    ref, _ = R.attention(_np(q), _np(k), _np(v), [(0, 1, 0, 3000), (1, 2, 3000, 5000)], 0, 0.125)
    _check("out", _np(out), *ref["out"], EPS["bf16"])
    del big


def test_bounds_are_clamped():
    """Bounds outside the rows, reversed, or longer than max_q and max_k reach no row that is not there."""
    torch = torch_cuda()
    announce("attention with bounds out of range")
    c = Case(dtype="bf16", lens=((40, 40), (30, 30), (20, 20)), heads=2, dim=64, mask=1, radius=5, seed=2)
    on = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    keep = [on(-5, 60, 70), on(40, 50, 2000000000), on(-5, 60, 70), on(40, 50, 2000000000)]
    for n, t in zip(("q_begin", "q_end", "k_begin", "k_end"), keep):
        setattr(c.a, n, t.data_ptr())
    c.run()
    c.spans = [(0, 40, 0, 40), (60, 60, 60, 60), (70, 90, 70, 90)]
    torch.cuda.synchronize()
    c.verify()


def test_gradient_against_differences():
    """fp32: the change of sum(out dout) along random directions, central differences with step 1e-2 (truncation about
    1e-4 of the value's scale, rounding about 1e-7 of sum |out dout| over the step): 1e-2 of the direction's scale."""
    torch = torch_cuda()
    announce("attention differences")
    kw = dict(dtype="f32", lens=((60, 60), (33, 33)), heads=4, kv_heads=2, dim=20, mask=1, cap=4.0, radius=10, p=0.2)
    c = Case(**kw)
    c.run()
    analytic = [t.double().clone() for t in c.grads] + [c.dtable.double().clone()]
    gen = torch.Generator(device="cuda").manual_seed(4)
    for t, grad in zip((c.q, c.k, c.v, c.table), analytic):
        d = torch.randn(t.shape, generator=gen, device="cuda")
        base, f = t.clone(), []
        for s in (1, -1):
            t.copy_(base + s * 1e-2 * d)
            A.fo_attn_fwd(c.a, c.q, c.k, c.v, c.out, None, c.ws)
            f.append(float((c.out.double() * c.dout.double()).sum()))
        t.copy_(base)
        want = float((grad * d.double()).sum())
        assert abs((f[0] - f[1]) / 2e-2 - want) <= 1e-2 * max(abs(want), float(grad.norm()))


# ------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,p,bias,res,pad", [
    (1, 1, 0.5, True, True, 0), (5, 7, 0.2, True, False, 0), (64, 100, 0.1, False, True, 0), (129, 768, 0.1, True, True, 0),
    (1000, 33, 0.25, True, True, 5), (3, 2304, 0.0, True, True, 0), (300, 100, 0.05, True, True, 1),
    (4097, 64, 0.1, True, False, 8), (70, 4100, 0.5, False, False, 4), (2, 8, 0.99999, False, False, 0)])
def test_dropout(dtype, rows, cols, p, bias, res, pad):
    """y and dx are one rounding of exact terms; dbias is a sum of rows of them (in fp32, then one rounding)."""
    torch = torch_cuda()
    announce(f"dropout {dtype} {rows}x{cols} p={p} bias={bias} residual={res} pad={pad}")
    dt, eps = _dt(dtype), {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}[dtype]  # unit roundoffs
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    mat = lambda: torch.randn((rows, cols + pad), generator=g, device="cuda").to(dt)[:, :cols]  # noqa: E731
    x, r, dy, y, dx = mat(), mat() if res else None, mat(), mat(), mat()
    b = torch.randn(cols, generator=g, device="cuda").to(dt) if bias else None
    db = torch.full((cols,), float("nan"), dtype=dt, device="cuda") if bias else None
    seed, off = (1 << 63) + 12345, 0xFFFFFFFE
    ws = torch.empty(A.fo_dropout_workspace(rows, cols), dtype=torch.uint8, device="cuda")
    A.fo_dropout_fwd(x, y, p, seed, off, bias=b, residual=r)
    A.fo_dropout_bwd(dy, dx, p, seed, off, dbias=db, workspace=ws)
    keep = R.drop_matrix(rows, cols, p, seed, off)
    xb = _np(x) + (_np(b) if bias else 0)
    want = xb * keep + (_np(r) if res else 0)
    # up to four fp32 roundings before the last one, relative to the parts they round
    slack = 4 * 2.0 ** -24 * (np.abs(xb * keep) + (np.abs(_np(r)) if res else 0) + (np.abs(_np(b)) if bias else 0) * keep)
    assert (np.abs(_np(y) - want) <= eps * np.abs(want) * 1.01 + slack).all()
    want = _np(dy) * keep
    assert (np.abs(_np(dx) - want) <= (1.01 * eps + 2.0 ** -23) * np.abs(want)).all()
    if bias:
        tot = np.abs(want).sum(0)
        assert (np.abs(_np(db) - want.sum(0)) <= eps * np.abs(want.sum(0)) * 1.01 + (np.sqrt(rows) + 4) * 2.0 ** -23 * tot).all()


def test_dropout_in_place_and_rate():
    torch = torch_cuda()
    announce("dropout in place 4096x768")
    x = torch.ones((4096, 768), dtype=torch.float32, device="cuda")
    r = torch.zeros_like(x)
    y = torch.empty_like(x)
    A.fo_dropout_fwd(x, y, 0.1, 3, 4, residual=r)
    A.fo_dropout_fwd(x, r, 0.1, 3, 4, residual=r)  # over the residual
    A.fo_dropout_fwd(x, x, 0.1, 3, 4)              # over the input
    assert torch.equal(x, y) and torch.equal(r, y)
    n = y.numel()
    share = float((y == 0).sum()) / n
    assert abs(share - 6554 / 65536) <= 5 * (0.09 / n) ** 0.5  # five standard deviations
    z = torch.ones_like(x)
    A.fo_dropout_fwd(z, z, 0.1, 3, 5)
    both = float(((z == 0) & (y == 0)).sum()) / n  # another offset: an independent mask
    assert abs(both - (6554 / 65536) ** 2) <= 5 * (0.01 / n) ** 0.5


def test_dropout_many_rows():
    """Element numbers past 2^32 (rows of 2^21 elements): the generator's second counter word is in use."""
    torch = torch_cuda()
    rows, cols = 2100, 1 << 21
    announce(f"dropout {rows}x{cols}")
    x = torch.ones((rows, cols), dtype=torch.bfloat16, device="cuda")
    A.fo_dropout_fwd(x, x, 0.5, 9, 1)
    n = np.uint64(2080) * np.uint64(cols // 8) + np.arange(64, dtype=np.uint64)
    h = R.halves(R.philox7(n & R.LOW, n >> np.uint64(32), 0, 1, 9)).reshape(-1)
    assert (_np(x[2080, :512]) == (h >= 32768) * 2.0).all()
    del x

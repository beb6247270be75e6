"""A language model's operators captured into HIP graphs, on other streams, and called again: the same bits."""
import numpy as np
import pytest

from tests.gpu_util import announce, torch_cuda

pytestmark = pytest.mark.gpu
A = pytest.importorskip("paper_2504_13850_amd.api")


def _calls(dtype, rows, cols, vocab):
    """Every operator on operands and results of its own, as functions of a stream; and what they write.  Workspaces
    are shared by all of them, as a program may that runs them one after the other."""
    torch = torch_cuda()
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    g = torch.Generator(device="cuda").manual_seed(rows)
    normal = lambda *s, t=dt: torch.randn(s, generator=g, device="cuda").to(t)  # noqa: E731
    new = lambda *s, t=dt: torch.full(s, float("nan"), dtype=t, device="cuda")  # noqa: E731
    f8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    f32 = torch.float32
    x = {"tokens": torch.randint(-1, vocab, (rows,), generator=g, device="cuda").to(torch.int32), "table": normal(vocab, cols),
         "x": normal(rows, cols), "res": normal(rows, cols), "w": normal(cols), "dy": normal(rows, cols),
         "logits": normal(rows, vocab), "weight": normal(rows, t=f32), "ref": normal(rows, t=f32)}
    cut = torch.tensor([0, rows // 3, rows // 2, rows - 1], dtype=torch.int32, device="cuda")
    begin, end = cut.contiguous(), torch.cat([cut[1:], cut[-1:] + 1]).contiguous()
    o = {"out": new(rows, cols), "dtable": new(vocab, cols), "h": new(rows, cols), "y": new(rows, cols), "rstd": new(rows, t=f32),
         "dx": new(rows, cols), "dw": new(cols), "y8": f8(rows, cols), "s8": new(rows, t=f32), "w8": f8(vocab, cols),
         "sw": new(vocab, t=f32), "c": new(rows, vocab), "logp": new(rows, t=f32), "lse": new(rows, t=f32),
         "dlogp": torch.zeros(rows, dtype=f32, device="cuda"), "loss": new(2, t=f32), "reward": new(4, t=f32),
         "dlogits": new(rows, vocab), "xent": new(rows, t=f32), "dxent": new(rows, vocab)}
    n = max(A.fo_embed_workspace(rows, cols, vocab), A.fo_rmsnorm_workspace(rows, cols), A.fo_logp_workspace(rows, vocab),
            A.fo_gemm_f8_workspace(rows, vocab, cols))
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")

    def run(s):
        A.fo_embed_fwd(x["tokens"], x["table"], o["out"], scale=3.0, stream=s)
        A.fo_embed_bwd(x["tokens"], x["dy"], o["dtable"], scale=3.0, workspace=ws, stream=s)
        A.fo_embed_bwd(x["tokens"], x["x"], o["dtable"], accumulate=True, workspace=ws, stream=s)
        A.fo_rmsnorm_fwd(x["x"], x["w"], o["y"], o["rstd"], 1e-6, residual=x["res"], h=o["h"], stream=s)
        A.fo_rmsnorm_bwd(x["dy"], o["h"], x["w"], o["rstd"], o["dx"], dw=o["dw"], dres=x["res"], workspace=ws, stream=s)
        A.fo_rmsnorm_f8(x["x"], x["w"], o["y8"], o["s8"], 1e-6, residual=x["res"], stream=s)
        A.fo_quant_f8(x["table"], o["w8"], o["sw"], stream=s)
        A.fo_gemm_f8(o["y8"], o["s8"], o["w8"], o["sw"], o["c"], workspace=ws, stream=s)
        A.fo_logp_fwd(x["logits"], x["tokens"], o["logp"], o["lse"], workspace=ws, stream=s)
        A.fo_pref_loss(o["logp"], x["ref"], begin, end, o["loss"], o["reward"], o["dlogp"], stream=s)
        A.fo_logp_bwd(x["logits"], x["tokens"], o["logp"], o["lse"], o["dlogp"], o["dlogits"], stream=s)
        A.fo_xent(x["logits"], x["tokens"], x["weight"], o["xent"], o["dxent"], workspace=ws, stream=s)

    return run, x, o


def _bits(o):
    torch = torch_cuda()
    return {n: t.view(torch.uint8).clone() for n, t in o.items()}


def _same(a, b):
    torch = torch_cuda()
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("dtype,rows,cols,vocab", [("bf16", 300, 96, 1000), ("f32", 37, 33, 129), ("bf16", 9000, 72, 3000),
                                                   ("f32", 40, 8208, 100), ("bf16", 3, 128, 30000)])
def test_captured_and_replayed(dtype, rows, cols, vocab):
    """Two graphs of all operators that share their workspace, replayed in turn with eager calls and other work between
    them, on operands that change: every replay gives the eager calls' bits."""
    torch = torch_cuda()
    announce(f"graphs, {dtype} {rows} x {cols}, vocab {vocab}")
    run, x, o = _calls(dtype, rows, cols, vocab)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(side)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(torch.cuda.current_stream())
        graphs.append(graph)
    for k in range(4):
        for n in ("x", "dy", "logits"):
            x[n].mul_(-1.25)
        x["tokens"].copy_(x["tokens"].roll(5 + k))
        run(torch.cuda.current_stream())
        torch.cuda.synchronize()
        want = _bits(o)
        for t in o.values():
            t.view(torch.uint8).fill_(0xA5) if t is not o["dlogp"] else t.zero_()
        torch.zeros(1 << 20, device="cuda").add_(1)  # other work
        graphs[k % 2].replay()
        graphs[(k + 1) % 2].replay()
        torch.cuda.synchronize()
        _same(want, _bits(o))


def test_two_streams():
    """The same calls on two streams at once, each with workspaces of its own, and again on the default stream."""
    torch = torch_cuda()
    announce("two streams")
    both = [_calls("bf16", 5000, 200, 2000) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for _ in range(3):
        for (run, _, _), s in zip(both, streams):
            run(s)
    torch.cuda.synchronize()
    first = _bits(both[0][2])
    _same(first, _bits(both[1][2]))
    both[0][0](None)
    torch.cuda.synchronize()
    _same(first, _bits(both[0][2]))


def test_calls_wait_for_their_stream():
    """A call on a stream runs behind that stream's work and before what follows it there."""
    torch = torch_cuda()
    announce("order on a stream")
    s = torch.cuda.Stream()
    x = torch.zeros((4096, 2048), device="cuda")
    y, rstd = torch.empty_like(x), torch.empty(4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(50):
            x.add_(0.02)
        A.fo_rmsnorm_fwd(x, None, y, rstd, 0.0, stream=s)
        x.fill_(float("nan"))
    torch.cuda.synchronize()
    assert np.abs(y.cpu().numpy() - 1).max() < 1e-5 and abs(float(rstd[17]) - 1) < 1e-5

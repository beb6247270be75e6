"""The preference model of examples/preference_lm.py: a language model's operators together, forward and backward."""
import importlib.util
import os

import numpy as np
import pytest

from tests.gpu_util import announce, torch_cuda

pytestmark = pytest.mark.gpu


def _example():
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "preference_lm.py")
    spec = importlib.util.spec_from_file_location("preference_lm", at)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _plain_logits(E, model, batch):
    """The model in torch at 64 bits, on the CPU: leaves and logits."""
    import torch
    leaves = [w.detach().double().cpu().requires_grad_() for w in model.parameters()]
    table, last, rest = leaves[0], leaves[1], iter(leaves[2:])
    blocks = [{n: next(rest) for n in b} for b in model.blocks]
    norm = lambda h, w: h * torch.rsqrt(h.square().mean(1, keepdim=True) + E.EPS) * w  # noqa: E731
    tokens, bounds = batch.tokens.long().cpu(), list(zip(batch.begin.tolist(), batch.end.tolist()))
    h = table[tokens] * E.WIDTH ** 0.5
    for b in blocks:
        q, k, v = [t.unflatten(1, (E.HEADS, E.DIM)).transpose(0, 1) for t in
                   (norm(h, b["norm1"]) @ b["qkv"].T).split(E.HEADS * E.DIM, 1)]
        out = []
        for lo, hi in bounds:
            s = q[:, lo:hi] @ k[:, lo:hi].transpose(1, 2) * E.DIM ** -0.5
            s = s.masked_fill(torch.ones(hi - lo, hi - lo, dtype=torch.bool).triu(1), -float("inf"))
            out.append((torch.softmax(s, -1) @ v[:, lo:hi]).transpose(0, 1).flatten(1))
        h = h + torch.cat(out) @ b["out"].T
        h = h + torch.nn.functional.gelu(norm(h, b["norm2"]) @ b["up"].T) @ b["down"].T
    return leaves, norm(h, last) @ table.T


def _plain_losses(E, logits, ref, batch):
    import torch
    t = batch.targets.long().cpu()
    logp = torch.where(t >= 0, torch.log_softmax(logits, 1).gather(1, t.clamp_min(0)[:, None])[:, 0], 0)
    r = torch.stack([E.BETA * (logp - ref)[lo:hi].sum() for lo, hi in zip(batch.answer.tolist(), batch.end.tolist())])
    d = r[0::2] - r[1::2]
    soft = torch.nn.functional.softplus
    pref = ((1 - E.SMOOTH) * soft(-d) + E.SMOOTH * soft(d)).mean()
    return -(logp * batch.weight.double().cpu()).sum(), pref, logp


def test_gradients():
    """One step of either loss in fp32 against the model in 64 bits, and that against differences.  A gradient passes
    through some twenty sums of up to 256 fp32 terms: 256 2^-24 of its norm each, 2^-11.6 in all; 2^-11 is asked.
    Central differences of the 64-bit loss along a direction, step 1e-5: 1e-6."""
    torch = torch_cuda()
    E = _example()
    model, rng = E.Model(torch.float32, seed=3), np.random.default_rng(5)
    batch = E.Batch(rng, 6)
    announce("preference model, gradients")
    ref = torch.from_numpy(-3 + 0.3 * rng.standard_normal(len(batch.tokens))).float().cuda()
    losses = (lambda: E.CrossEntropy.apply(model.logits(batch.tokens, batch), batch.targets, batch.weight),
              lambda: E.preference_loss(model, ref, batch)[0])
    for which, f in enumerate(losses):
        loss = f()
        got = torch.autograd.grad(loss, model.parameters())
        leaves, logits = _plain_logits(E, model, batch)
        want = _plain_losses(E, logits, ref.double().cpu(), batch)[which]
        assert abs(float(loss) - float(want)) <= 2 ** -16 * abs(float(want))
        grads = torch.autograd.grad(want, leaves)
        for i, (g, w) in enumerate(zip(got, grads)):
            assert float((g.double().cpu() - w).norm()) <= 2 ** -11 * float(w.norm()), (which, i)
        # against differences of the 64-bit loss
        step = [torch.from_numpy(rng.standard_normal(tuple(w.shape))) for w in leaves]
        at = []
        with torch.no_grad():
            for s in (1e-5, -1e-5):
                for p, w, d in zip(model.parameters(), leaves, step):
                    p.data = w.detach() + s * d
                at.append(float(_plain_losses(E, _plain_logits(E, model, batch)[1], ref.double().cpu(), batch)[which]))
                for p, w in zip(model.parameters(), leaves):
                    p.data = w.detach().float().cuda()
        want = float(sum((g * d).sum() for g, d in zip(grads, step)))
        assert abs((at[0] - at[1]) / 2e-5 - want) <= 1e-6 * max(1.0, abs(want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_frozen_model(dtype):
    """The 8-bit copy's logits against the model in 64 bits.  A rounding to e4m3 is off by 2^-4 of a value at most, 2.6%
    in the root mean square; a product rounds both operands, and nine products follow each other: 3.7% sqrt(9) = 11% of
    the logits' norm where errors are independent, twice that is asked."""
    torch = torch_cuda()
    announce(f"preference model, frozen copy, {dtype}")
    E = _example()
    model = E.Model({"f32": torch.float32, "bf16": torch.bfloat16}[dtype], seed=4)
    batch = E.Batch(np.random.default_rng(6), 20)
    frozen = E.Frozen(model)
    got = frozen.logits(batch.tokens, batch).double().cpu()
    want = _plain_logits(E, model, batch)[1].detach()
    assert float((got - want).norm()) <= 0.22 * float(want.norm())
    logp = frozen.logp(batch.tokens, batch.targets, batch).double().cpu()
    t = batch.targets.long().cpu()
    same = torch.where(t >= 0, torch.log_softmax(got, 1).gather(1, t.clamp_min(0)[:, None])[:, 0], 0)
    assert float((logp - same).abs().max()) <= 2 ** -18 * float(same.abs().max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_runs_and_runs_the_same(dtype):
    """Both phases run; twice the same weights where torch's own kernels keep their order: the operators add none."""
    torch = torch_cuda()
    announce(f"preference model, {dtype}, twice")
    E = _example()
    torch.use_deterministic_algorithms(True, warn_only=True)
    try:
        a, b = (E.train(6, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype], say=lambda *_, **__: None)[0]
                for _ in range(2))
    finally:
        torch.use_deterministic_algorithms(False)
    for x, y in zip(a.parameters(), b.parameters()):
        assert bool(x.isfinite().all()) and torch.equal(x, y)

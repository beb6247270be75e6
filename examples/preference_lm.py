"""A small causal language model on the library's operators, trained on answers in pairs: the chosen one of each pair
against the rejected one, beside a frozen copy of the model that is evaluated in 8 bits.

    python examples/preference_lm.py [--steps 60] [--dtype f32|bf16]

Every prompt is a row of random tokens; the chosen answer repeats it, the rejected one is random.  First the model
learns answers of either kind by cross-entropy, then the preference.  Embedding, norms with the residual's addition,
attention, cross-entropy, log probabilities and the preference loss are the library's calls, forward and backward, and
the frozen copy's products are of 8-bit rows; the rest is torch.
"""
import argparse
import os
import sys

import numpy as np
import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2504_13850_amd import api as A  # noqa: E402

VOCAB, WIDTH, HEADS, DIM, LAYERS, PROMPT, ANSWER = 48, 128, 4, 32, 2, 8, 12
EPS, BETA, SMOOTH = 1e-6, 0.2, 0.05


def scratch(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def floats(n):
    return torch.empty(n, dtype=torch.float32, device="cuda")


def now():
    return torch.cuda.current_stream()


# ------------------------------------------------------------------ the operators as autograd knows them
class Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, table, scale):
        out = torch.empty((len(tokens), table.shape[1]), dtype=table.dtype, device="cuda")
        A.fo_embed_fwd(tokens, table, out, scale=scale, stream=now())
        ctx.save_for_backward(tokens)
        ctx.rest = table.shape, scale
        return out

    @staticmethod
    def backward(ctx, dout):
        (tokens,), (shape, scale) = ctx.saved_tensors, ctx.rest
        dtable = torch.empty(shape, dtype=dout.dtype, device="cuda")
        ws = scratch(A.fo_embed_workspace(len(tokens), shape[1], shape[0]))
        A.fo_embed_bwd(tokens, dout.contiguous(), dtable, scale=scale, workspace=ws, stream=now())
        return None, dtable, None


class AddNorm(torch.autograd.Function):
    """h = x + residual and its norm; both go on."""

    @staticmethod
    def forward(ctx, x, residual, w):
        h, y, rstd = torch.empty_like(x), torch.empty_like(x), floats(len(x))
        A.fo_rmsnorm_fwd(x, w, y, rstd, EPS, residual=residual, h=h, stream=now())
        ctx.save_for_backward(h, w, rstd)
        return h, y

    @staticmethod
    def backward(ctx, dh, dy):
        h, w, rstd = ctx.saved_tensors
        dx, dw, ws = torch.empty_like(h), torch.empty_like(w), scratch(A.fo_rmsnorm_workspace(*h.shape))
        A.fo_rmsnorm_bwd(dy.contiguous(), h, w, rstd, dx, dw, dres=dh.contiguous(), workspace=ws, stream=now())
        return dx, dx, dw


class Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, seq):
        out, a, lse, ws = attention(qkv, seq, True)
        ctx.save_for_backward(qkv, out, lse)
        ctx.rest = a, ws, seq  # the record holds addresses of the bounds
        return out

    @staticmethod
    def backward(ctx, dout):
        qkv, out, lse = ctx.saved_tensors
        a, ws, _ = ctx.rest
        dqkv = torch.empty_like(qkv)
        A.fo_attn_bwd(a, *split(qkv), out, lse, dout.contiguous(), *split(dqkv), None, ws, stream=now())
        return dqkv, None


class LogProb(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets):
        logp, lse = floats(len(logits)), floats(len(logits))
        A.fo_logp_fwd(logits, targets, logp, lse, workspace=scratch(A.fo_logp_workspace(*logits.shape)), stream=now())
        ctx.save_for_backward(logits, targets, logp, lse)
        return logp

    @staticmethod
    def backward(ctx, dlogp):
        logits, targets, logp, lse = ctx.saved_tensors
        dlogits = torch.empty_like(logits)
        A.fo_logp_bwd(logits, targets, logp, lse, dlogp.contiguous(), dlogits, stream=now())
        return dlogits, None


class CrossEntropy(torch.autograd.Function):
    """The weighted sum of the rows' losses; their gradient is made with them."""

    @staticmethod
    def forward(ctx, logits, targets, weight):
        loss, dlogits = floats(len(logits)), torch.empty_like(logits)
        ws = scratch(A.fo_logp_workspace(*logits.shape))
        A.fo_xent(logits, targets, weight, loss, dlogits, workspace=ws, stream=now())
        ctx.save_for_backward(dlogits)
        return loss @ weight

    @staticmethod
    def backward(ctx, dloss):
        return ctx.saved_tensors[0] * dloss.to(ctx.saved_tensors[0].dtype), None, None


class Preference(torch.autograd.Function):
    """The mean loss over the pairs, and the answers' rewards."""

    @staticmethod
    def forward(ctx, logp, ref, begin, end):
        pairs = len(begin) // 2
        loss, reward, dlogp = floats(pairs), floats(2 * pairs), torch.zeros_like(logp)
        A.fo_pref_loss(logp, ref, begin, end, loss, reward, dlogp, beta=BETA, smooth=SMOOTH, dloss=1.0 / pairs,
                       stream=now())
        ctx.save_for_backward(dlogp)
        ctx.mark_non_differentiable(reward)
        return loss.mean(), reward

    @staticmethod
    def backward(ctx, dloss, _):
        return ctx.saved_tensors[0] * dloss, None, None, None


def split(qkv):
    return [t.unflatten(1, (HEADS, DIM)) for t in qkv.split(HEADS * DIM, 1)]


def attention(qkv, seq, train):
    q, k, v = split(qkv)
    out = torch.empty((len(qkv), HEADS, DIM), dtype=qkv.dtype, device="cuda")
    lse = torch.empty((HEADS, len(qkv)), dtype=torch.float32, device="cuda") if train else None
    a = A.make_attn(q, k, v, out, seq.begin, seq.end, seq.begin, seq.end, seq.most, seq.most, mask=A.FO_ATTN_CAUSAL)
    ws = scratch(A.fo_attn_workspace(a, train))
    A.fo_attn_fwd(a, q, k, v, out, lse, ws, stream=now())
    return out, a, lse, ws


# ------------------------------------------------------------------ the model
class Model:
    def __init__(self, dtype, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def mat(*shape, scale=None):
            s = shape[1] ** -0.5 if scale is None else scale
            return (torch.randn(shape, generator=g, device="cuda") * s).to(dtype).requires_grad_()

        def ones():
            return torch.ones(WIDTH, dtype=dtype, device="cuda", requires_grad=True)

        # weights are [outputs][inputs]; the embedding's table is the output's weights too
        self.table = mat(VOCAB, WIDTH, scale=0.1)
        self.last = ones()
        self.blocks = [{"qkv": mat(3 * HEADS * DIM, WIDTH), "out": mat(WIDTH, HEADS * DIM), "up": mat(2 * WIDTH, WIDTH),
                        "down": mat(WIDTH, 2 * WIDTH), "norm1": ones(), "norm2": ones()} for _ in range(LAYERS)]

    def parameters(self):
        return [self.table, self.last] + [w for b in self.blocks for w in b.values()]

    def logits(self, tokens, seq):
        h, add = Embed.apply(tokens, self.table, WIDTH ** 0.5), None
        for b in self.blocks:
            add = torch.zeros_like(h) if add is None else add
            h, y = AddNorm.apply(h, add, b["norm1"])
            h, y = AddNorm.apply(h, Attention.apply(y @ b["qkv"].T, seq).flatten(1) @ b["out"].T, b["norm2"])
            add = F.gelu(y @ b["up"].T) @ b["down"].T
        return AddNorm.apply(h, add, self.last)[1] @ self.table.T


class Frozen:
    """A model's copy for passes without a gradient: weights and the products' operands in 8 bits."""

    def __init__(self, model):
        self.table, self.last = model.table.detach().clone(), model.last.detach().clone()
        self.head = self.eight(self.table)
        self.blocks = [{n: w.detach().clone() if n.startswith("norm") else self.eight(w.detach()) for n, w in b.items()}
                       for b in model.blocks]

    @staticmethod
    def eight(x):
        q, scale = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda"), floats(len(x))
        A.fo_quant_f8(x, q, scale, stream=now())
        return q, scale

    def product(self, a, b):
        c = torch.empty((len(a[0]), len(b[0])), dtype=self.table.dtype, device="cuda")
        ws = scratch(A.fo_gemm_f8_workspace(len(a[0]), len(b[0]), a[0].shape[1]))
        A.fo_gemm_f8(*a, *b, c, workspace=ws, stream=now())
        return c

    @staticmethod
    def norm(x, residual, w):
        h, q, scale = torch.empty_like(x), torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda"), floats(len(x))
        A.fo_rmsnorm_f8(x, w, q, scale, EPS, residual=residual, h=h, stream=now())
        return h, (q, scale)

    @torch.no_grad()
    def logits(self, tokens, seq):
        h = torch.empty((len(tokens), WIDTH), dtype=self.table.dtype, device="cuda")
        A.fo_embed_fwd(tokens, self.table, h, scale=WIDTH ** 0.5, stream=now())
        add = None
        for b in self.blocks:
            h, y = self.norm(h, add, b["norm1"])
            o = attention(self.product(y, b["qkv"]), seq, False)[0]
            h, y = self.norm(h, self.product(self.eight(o.flatten(1)), b["out"]), b["norm2"])
            add = self.product(self.eight(F.gelu(self.product(y, b["up"]))), b["down"])
        return self.product(self.norm(h, add, self.last)[1], self.head)

    @torch.no_grad()
    def logp(self, tokens, targets, seq):
        logits = self.logits(tokens, seq)
        logp = floats(len(logits))
        A.fo_logp_fwd(logits, targets, logp, workspace=scratch(A.fo_logp_workspace(*logits.shape)), stream=now())
        return logp


class Batch:
    """Pairs of sequences, prompt and answer, one after the other; targets are the next tokens, -1 in the prompts."""

    def __init__(self, rng, pairs):
        rows, targets, spans, at = [], [], [], 0
        for _ in range(pairs):
            prompt = rng.integers(0, VOCAB, PROMPT)
            for chosen in (True, False):
                n = int(rng.integers(3, ANSWER + 1))
                answer = np.resize(prompt, n) if chosen else rng.integers(0, VOCAB, n)
                whole = np.concatenate([prompt, answer])
                rows.append(whole[:-1])
                targets.append(np.where(np.arange(len(whole) - 1) < PROMPT - 1, -1, whole[1:]))
                spans.append((at, at + PROMPT - 1, at + len(whole) - 1))
                at += len(whole) - 1
        i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
        self.tokens, self.targets = i32(np.concatenate(rows)), i32(np.concatenate(targets))
        self.begin, self.answer, self.end = (i32([s[k] for s in spans]) for k in range(3))
        self.most = max(s[2] - s[0] for s in spans)
        answers = int(sum(s[2] - s[1] for s in spans))
        self.weight = torch.full((at,), 1.0 / answers, device="cuda")


def preference_loss(model, ref, batch):
    logp = LogProb.apply(model.logits(batch.tokens, batch), batch.targets)
    return Preference.apply(logp, ref, batch.answer, batch.end)


def train(steps, dtype, say=print):
    model, rng = Model(dtype), np.random.default_rng(1)
    opt = torch.optim.Adam(model.parameters(), lr=2e-3)
    for step in range(steps):
        b = Batch(rng, 32)
        loss = CrossEntropy.apply(model.logits(b.tokens, b), b.targets, b.weight)
        opt.zero_grad()
        loss.backward()
        opt.step()
        if step % 20 == 0 or step == steps - 1:
            say(f"cross-entropy, step {step}: {float(loss.detach()):.3f}", flush=True)
    frozen = Frozen(model)
    for step in range(steps):
        b = Batch(rng, 32)
        loss, reward = preference_loss(model, frozen.logp(b.tokens, b.targets, b), b)
        opt.zero_grad()
        loss.backward()
        opt.step()
        if step % 20 == 0 or step == steps - 1:
            ahead = (reward[0::2] > reward[1::2]).float().mean()
            say(f"preference, step {step}: {float(loss.detach()):.3f}, chosen ahead in {float(ahead):.0%}", flush=True)
    return model, frozen


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dtype", choices=["f32", "bf16"], default="f32")
    a = ap.parse_args()
    train(a.steps, {"f32": torch.float32, "bf16": torch.bfloat16}[a.dtype])


if __name__ == "__main__":
    main()

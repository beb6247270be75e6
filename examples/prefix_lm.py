"""A small prefix language model on the transformer operators: training on packed
sequences, then generation token by token against a cache of keys and values.

    python examples/prefix_lm.py [--steps 200] [--dtype f32|bf16]

Every sequence repeats a random pattern of eight tokens; the first eight are its
prefix, whose tokens all see each other, and the model learns to go on.  Attention
(prefix mask, capped scores, learned bias by distance, dropout of the
probabilities, key heads shared by two) and the sublayers' dropout with bias and
residual are the library's calls, forward and backward; the rest is torch.
"""
import argparse
import os
import sys

import numpy as np
import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2504_13850_amd import api as A  # noqa: E402

VOCAB, WIDTH, HEADS, KV, DIM, LAYERS, PERIOD = 32, 128, 4, 2, 32, 2, 8
BUCKETS, RADIUS, CAP, SEED = 16, 64, 30.0, 2024


class Packed:
    """Row bounds of sequences that lie one after the other, for queries and keys alike."""

    def __init__(self, lens, prefix):
        cu = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
        self.begin, self.end, self.most = cu[:-1], cu[1:], max(lens)
        self.prefix = torch.tensor(prefix, dtype=torch.int32, device="cuda")


def split(qkv):
    """q, k and v as columns of the fused projection's rows, without a copy."""
    return [t.unflatten(1, (-1, DIM)) for t in qkv.split((HEADS * DIM, KV * DIM, KV * DIM), 1)]


class Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, table, bucket, seq, p, offset):
        q, k, v = split(qkv)
        out = torch.empty((len(qkv), HEADS, DIM), dtype=qkv.dtype, device="cuda")
        lse = torch.empty((HEADS, len(qkv)), dtype=torch.float32, device="cuda")
        a = A.make_attn(q, k, v, out, seq.begin, seq.end, seq.begin, seq.end, seq.most, seq.most, cap=CAP,
                        mask=A.FO_ATTN_PREFIX, prefix=seq.prefix, table=table, bucket=bucket, p=p, seed=SEED,
                        offset=offset)
        ws = torch.empty(A.fo_attn_workspace(a, True), dtype=torch.uint8, device="cuda")
        A.fo_attn_fwd(a, q, k, v, out, lse, ws, stream=torch.cuda.current_stream())
        ctx.save_for_backward(qkv, table, bucket, out, lse)
        ctx.rest = a, ws, seq  # the record holds addresses of the bounds
        return out

    @staticmethod
    def backward(ctx, dout):
        qkv, table, bucket, out, lse = ctx.saved_tensors
        a, ws, _ = ctx.rest
        dqkv, dtable = torch.empty_like(qkv), torch.empty_like(table)
        A.fo_attn_bwd(a, *split(qkv), out, lse, dout.contiguous(), *split(dqkv), dtable, ws,
                      stream=torch.cuda.current_stream())
        return dqkv, dtable, None, None, None, None


class DropAdd(torch.autograd.Function):
    """dropout(x + bias) + residual; the backward pass draws the mask again."""

    @staticmethod
    def forward(ctx, x, bias, residual, p, offset):
        y = torch.empty_like(x)
        A.fo_dropout_fwd(x, y, p, SEED, offset, bias=bias, residual=residual, stream=torch.cuda.current_stream())
        ctx.rest = p, offset
        return y

    @staticmethod
    def backward(ctx, dy):
        dy = dy.contiguous()
        dx, dbias = torch.empty_like(dy), torch.empty(dy.shape[1], dtype=dy.dtype, device="cuda")
        ws = torch.empty(A.fo_dropout_workspace(*dy.shape), dtype=torch.uint8, device="cuda")
        A.fo_dropout_bwd(dy, dx, ctx.rest[0], SEED, ctx.rest[1], dbias=dbias, workspace=ws,
                         stream=torch.cuda.current_stream())
        return dx, dbias, dy, None, None


class PrefixLM:
    def __init__(self, dtype, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def mat(*shape, scale):
            return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype).requires_grad_()

        def zeros(*shape):
            return torch.zeros(shape, dtype=dtype, device="cuda", requires_grad=True)

        self.embed = mat(VOCAB, WIDTH, scale=1.0)
        self.head = mat(WIDTH, VOCAB, scale=WIDTH ** -0.5)
        self.blocks = [{"qkv": mat(WIDTH, (HEADS + 2 * KV) * DIM, scale=WIDTH ** -0.5),
                        "out": mat(HEADS * DIM, WIDTH, scale=WIDTH ** -0.5), "out_b": zeros(WIDTH),
                        "up": mat(WIDTH, 2 * WIDTH, scale=WIDTH ** -0.5),
                        "down": mat(2 * WIDTH, WIDTH, scale=WIDTH ** -0.5), "down_b": zeros(WIDTH),
                        "bias": zeros(BUCKETS, HEADS)} for _ in range(LAYERS)]
        self.bucket = torch.from_numpy(A.fo_relpos_buckets(BUCKETS, RADIUS, True)).cuda()

    def parameters(self):
        return [self.embed, self.head] + [w for b in self.blocks for w in b.values()]

    def forward(self, tokens, attend, p=0.0, step=0):
        """Logits of every row.  attend(layer, qkv, table, offset) -> [rows, heads, dim]."""
        x = self.embed[tokens]
        for n, b in enumerate(self.blocks):
            at = 3 * (step * LAYERS + n)  # another offset for each dropout of each step
            o = attend(n, F.layer_norm(x, (WIDTH,)) @ b["qkv"], b["bias"], at)
            x = DropAdd.apply(o.flatten(1) @ b["out"], b["out_b"], x, p, at + 1)
            u = F.gelu(F.layer_norm(x, (WIDTH,)) @ b["up"])
            x = DropAdd.apply(u @ b["down"], b["down_b"], x, p, at + 2)
        return F.layer_norm(x, (WIDTH,)) @ self.head

    def packed(self, tokens, seq, p=0.0, step=0):
        return self.forward(tokens, lambda n, qkv, table, at: Attention.apply(qkv, table, self.bucket, seq, p, at), p,
                            step)


def batch(rng, n):
    """Packed tokens of n sequences, the rows whose next token follows from the pattern, and those tokens."""
    lens = [int(v) for v in rng.integers(2 * PERIOD, 64, n)]
    rows = [np.resize(rng.integers(0, VOCAB, PERIOD), m) for m in lens]
    at = np.concatenate(([0], np.cumsum(lens)))
    known = np.concatenate([np.arange(at[i] + PERIOD - 1, at[i + 1] - 1) for i in range(n)])
    tokens = np.concatenate(rows)
    on = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    return on(tokens), Packed(lens, [PERIOD] * n), on(known), on(tokens[known + 1])


def train(steps, dtype, say=print):
    model, rng = PrefixLM(dtype), np.random.default_rng(1)
    opt = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses = []
    for step in range(steps):
        tokens, seq, known, want = batch(rng, 32)
        loss = F.cross_entropy(model.packed(tokens, seq, 0.1, step)[known].float(), want)
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
        if step % 50 == 0 or step == steps - 1:
            say(f"step {step}: loss {losses[-1]:.3f}", flush=True)
    return model, losses


@torch.no_grad()
def generate(model, prompts, count):
    """`count` tokens after each prompt [n, PERIOD], and the logits of every row they were chosen from."""
    n, room, dtype = len(prompts), PERIOD + count, model.embed.dtype
    cache = [torch.empty((2, n * room, KV, DIM), dtype=dtype, device="cuda") for _ in range(LAYERS)]
    i32 = lambda v: torch.as_tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    begin, length = torch.arange(n, device="cuda", dtype=torch.int32) * room, 0
    prefix = i32([PERIOD] * n)
    tokens, got, logits = prompts.flatten(), [], []
    for _ in range(count):
        new = len(tokens) // n  # the prompt's tokens, then one
        rows = (begin.long()[:, None] + torch.arange(length, length + new, device="cuda")).flatten()
        length += new
        q_begin, k_end = torch.arange(n, device="cuda", dtype=torch.int32) * new, begin + length
        q_end = q_begin + new

        def attend(layer, qkv, table, at):
            q, k, v = split(qkv)
            kc, vc = cache[layer]
            kc[rows], vc[rows] = k, v
            out = torch.empty((len(qkv), HEADS, DIM), dtype=dtype, device="cuda")
            a = A.make_attn(q, kc, vc, out, q_begin, q_end, begin, k_end, new, length, cap=CAP, mask=A.FO_ATTN_PREFIX,
                            prefix=prefix, table=table, bucket=model.bucket)
            ws = torch.empty(A.fo_attn_workspace(a), dtype=torch.uint8, device="cuda")
            A.fo_attn_fwd(a, q, kc, vc, out, None, ws, stream=torch.cuda.current_stream())
            return out

        logits.append(model.forward(tokens, attend).view(n, new, VOCAB)[:, -1])
        tokens = logits[-1].argmax(-1)
        got.append(tokens)
    return torch.stack(got, 1), torch.stack(logits, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--dtype", choices=["f32", "bf16"], default="f32")
    a = ap.parse_args()
    model, _ = train(a.steps, {"f32": torch.float32, "bf16": torch.bfloat16}[a.dtype])
    prompts = torch.randint(0, VOCAB, (4, PERIOD), generator=torch.Generator().manual_seed(5)).cuda()
    got, _ = generate(model, prompts, 2 * PERIOD)
    for p, t in zip(prompts.tolist(), got.tolist()):
        print(p, "->", t)
    right = (got == prompts.repeat(1, 2)).float().mean()
    print(f"tokens that continue the pattern: {float(right):.0%}")


if __name__ == "__main__":
    main()

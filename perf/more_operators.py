"""The operators of a language model's step around its attention, as cases to time and to check.

Each kind goes through the public binding (paper_2504_13850_amd.api):

  embed   rows of a table by tokens, and the table's gradient
  norm    root-mean-square norm with the residual's addition, forward and backward
  norm8   the same forward with an 8-bit (e4m3) output and a scale a row, as a pass without gradients has it
  quant8  rows to 8 bits with a scale each, without a norm (weights, other activations)
  gemm8   the product of two matrices of 8-bit rows with scales
  logp    log probabilities of target tokens: "train" the cross-entropy with its gradient, else the forward pass
  pref    a preference loss on the log probabilities of answers in pairs, with its gradient
  step    the whole of it: log probabilities from logits, the preference loss, the logits' gradient

``own`` False computes them in plain torch at 32 bits, True calls the library.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
F8 = torch.float8_e4m3fn
F8_MAX = 448.0
EPS = 1e-6


def listed():
    embed = {"kind": "embed", "dtype": "bf16", "zipf": 1.0, "pad": 0.0, "scale": 1.0}
    norm = {"kind": "norm", "dtype": "bf16", "residual": True}
    gemm = {"kind": "gemm8", "dtype": "bf16"}
    pref = {"dtype": "bf16", "beta": 0.1, "smooth": 0.0, "mean": False, "lens_seed": 1}
    return [
        # the BERT-shaped encoder's batch of 32 sequences, an ordinary subword vocabulary with its frequent tokens
        dict(embed, name="embed_bert_4k", rows=4096, vocab=32000, cols=768),
        # a language model's large packed batch, a tenth of it padding
        dict(embed, name="embed_docs_64k", rows=65536, vocab=128000, cols=2048, pad=0.1, scale=45.25),
        # between the sublayers of the BERT-shaped encoder
        dict(norm, name="norm_bert_4k", rows=4096, cols=768),
        # the same of a wide model with a large batch
        dict(norm, name="norm_docs_16k", rows=16384, cols=4096),
        # a frozen model's pass over a ragged batch: the next product's 8-bit operand
        dict(norm, name="norm8_docs_8k", kind="norm8", rows=8191, cols=4096),
        # single tokens of four sequences through one projection: the weights are read for four rows
        dict(gemm, name="gemm8_one", m=4, n=4096, k=4096),
        # the BERT-shaped encoder's fused projection on a ragged batch
        dict(gemm, name="gemm8_bert_qkv", m=2603, n=2304, k=768),
        # the largest: a wide model's projection over a long batch
        dict(gemm, name="gemm8_docs_8k", m=8192, n=8192, k=8192),
        # cross-entropy of a packed batch, some of its rows without a target
        dict(kind="logp", name="xent_docs_8k", dtype="bf16", rows=8192, vocab=32000, train=True, scale=1.0, ignore=0.1),
        # log probabilities of the tokens just drawn for five sequences, large vocabulary
        dict(kind="logp", name="logp_one", dtype="f32", rows=5, vocab=128000, train=False, scale=1.0, ignore=0.0),
        # the loss alone, as a program has it that keeps the log probabilities
        dict(pref, kind="pref", name="pref_64", pairs=64, min_len=50, max_len=1000),
        # a step from logits to their gradient: eight pairs of answers
        dict(pref, kind="step", name="step_8", pairs=8, min_len=100, max_len=600, vocab=32000, smooth=0.1),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {"flops": 0.0, "bytes": 0.0}
    for c in listed():
        most = {k: max(v, work(c)[k]) for k, v in most.items()}
    kind = rng.choice(["embed", "embed", "norm", "norm", "norm8", "quant8", "gemm8", "gemm8", "logp", "logp", "pref", "step"])
    case = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if kind == "embed":
        case.update(rows=_log_int(rng, 1, 65536), vocab=_log_int(rng, 2, 128000), cols=_log_int(rng, 8, 4096),
                    zipf=rng.choice([0.0, 1.0]), pad=rng.choice([0.0, 0.1]), scale=rng.choice([1.0, 11.5]))
        cut = "rows" if case["rows"] > case["vocab"] else "vocab"
    elif kind in ("norm", "norm8", "quant8"):
        case.update(rows=_log_int(rng, 1, 16384), cols=_log_int(rng, 8, 16384),
                    residual=kind != "quant8" and rng.random() < 0.7)
        cut = "rows"
    elif kind == "gemm8":
        size = lambda step: max(1, round(_log_int(rng, 1, 8192) / step) * step)  # noqa: E731
        case.update(m=_log_int(rng, 1, 8192), n=size(rng.choice([1, 16, 256])),
                    k=max(8, size(rng.choice([1, 16, 64, 256]))))
        cut = "m"
    elif kind == "logp":
        case.update(rows=_log_int(rng, 1, 8192), vocab=_log_int(rng, 4, 128000), train=rng.random() < 0.6,
                    scale=rng.choice([1.0, 0.7]), ignore=rng.choice([0.0, 0.3]))
        cut = "rows"
    else:
        hi = _log_int(rng, 2, 2000)
        case.update(pairs=_log_int(rng, 1, 128), min_len=max(1, int(hi * rng.uniform(0.1, 1.0))), max_len=hi,
                    lens_seed=rng.randint(1, 1000), beta=rng.choice([0.05, 0.1, 0.5]), smooth=rng.choice([0.0, 0.1]),
                    mean=rng.random() < 0.3)
        if kind == "step":
            case["vocab"] = _log_int(rng, 8, 64000)
        cut = "pairs"
    while any(work(case)[k] > most[k] for k in most):
        if case[cut] > 1:
            case[cut] //= 2
        else:
            case["max_len"] = max(1, case["max_len"] // 2)
            case["min_len"] = min(case["min_len"], case["max_len"])
    return case


# ------------------------------------------------------------------ what a case holds
def _shares(case):
    """How often each token of the vocabulary comes: by rank, or all alike."""
    w = 1.0 / (np.arange(case["vocab"]) + 3.0) ** case["zipf"]
    return w / w.sum()


def _lens(case):
    """Rows of each answer (chosen and rejected in turn), the same for every seed."""
    r = random.Random(case["lens_seed"])
    return [r.randint(case["min_len"], case["max_len"]) for _ in range(2 * case["pairs"])]


def work(case):
    size, kind = 2 if case["dtype"] == "bf16" else 4, case["kind"]
    if kind == "embed":
        n = case["rows"] * (1 - case["pad"])
        found = float((1 - (1 - _shares(case)) ** n).sum())  # rows of the table that some token names
        # those in, out out; out's gradient in, the table's out; the tokens
        return {"bytes": (found + 2 * case["rows"] + case["vocab"]) * case["cols"] * size + 4.0 * case["rows"],
                "flops": 0.0}
    if kind == "gemm8":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": float((m + n) * (k + 4) + m * n * size), "flops": 2.0 * m * n * k}
    if kind == "logp":
        n = float(case["rows"]) * case["vocab"] * size
        return {"bytes": (2 if case["train"] else 1) * n + 16.0 * case["rows"], "flops": 0.0}
    if kind in ("pref", "step"):
        t = float(sum(_lens(case)))
        return {"bytes": 12.0 * t + (2 * t * case["vocab"] * size if kind == "step" else 0.0), "flops": 0.0}
    n = float(case["rows"]) * case["cols"]
    r = 1 if case["residual"] else 0
    if kind == "norm":  # x, residual in, h and y out; dy, h and h's other gradient in, dx out
        return {"bytes": n * size * (2 + 2 * r + 3 + r), "flops": 0.0}
    return {"bytes": n * (size * (1 + 2 * r) + 1), "flops": 0.0}  # x, residual in, h and 8 bits out


def _quantised(x):
    """Rows in 8 bits and their scales."""
    s = x.abs().amax(1) / F8_MAX
    return (x / s.clamp_min(1e-30)[:, None]).to(F8), s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, kind = DT[case["dtype"]], case["kind"]

    def normal(*shape, scale=1.0, to=None):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(to or dt)

    def ints(n, below):
        return torch.randint(0, below, (n,), generator=g, device="cuda")

    s = {"case": case}
    if kind == "embed":
        r, v, c = case["rows"], case["vocab"], case["cols"]
        up = torch.from_numpy(np.cumsum(_shares(case))).cuda()
        at = torch.searchsorted(up, torch.rand(r, generator=g, device="cuda", dtype=torch.float64)).clamp_max(v - 1)
        name = torch.randperm(v, generator=g, device="cuda")  # frequent tokens stand anywhere
        tokens = name[at].to(torch.int32)
        if case["pad"]:  # rows of padding hold no token
            tokens[1:][torch.rand(r - 1, generator=g, device="cuda") < case["pad"]] = -1
        s.update(tokens=tokens, table=normal(v, c, scale=0.05), dout=normal(r, c))
    elif kind == "gemm8":
        a, b = normal(case["m"], case["k"], to=torch.float32), normal(case["n"], case["k"], to=torch.float32, scale=0.02)
        (qa, sa), (qb, sb) = _quantised(a), _quantised(b)
        s.update(a=qa, a_scale=sa, b=qb, b_scale=sb)
    elif kind in ("norm", "norm8", "quant8"):
        r, c = case["rows"], case["cols"]
        s.update(x=normal(r, c), residual=normal(r, c, scale=2.0) if case["residual"] else None,
                 w=(1 + normal(c, scale=0.2, to=torch.float32)).to(dt))
        if kind == "norm":
            s.update(dy=normal(r, c), dres=normal(r, c) if case["residual"] else None)
    else:
        if kind == "logp":
            rows = case["rows"]
        else:
            lens = _lens(case)
            at = np.concatenate([[0], np.cumsum(lens)])
            rows = int(at[-1])
            s.update(begin=torch.from_numpy(at[:-1].astype(np.int32)).cuda(),
                     end=torch.from_numpy(at[1:].astype(np.int32)).cuda())
        if kind == "pref":
            logp = -normal(rows, to=torch.float32).abs() * 2
            s["logp"] = logp
        else:
            # a trained model's logits: many alike, and the right token ahead of them more often than not
            logits, targets = normal(rows, case["vocab"], scale=1.5, to=torch.float32), ints(rows, case["vocab"])
            logits[torch.arange(rows, device="cuda"), targets] += 4 + 3 * torch.randn(rows, generator=g, device="cuda")
            s["logits"], s["targets"] = logits.to(dt), targets.to(torch.int32)
            logp = logits[torch.arange(rows, device="cuda"), targets] - logits.logsumexp(1)
        if kind == "logp":
            if case["ignore"]:
                s["targets"][1:][torch.rand(rows - 1, generator=g, device="cuda") < case["ignore"]] = -1
            if case["train"]:  # each row's share of the mean over the rows that have a target
                s["weight"] = torch.full((rows,), 1.0 / rows, device="cuda")
        else:  # the frozen model's: the trained one has moved towards the chosen answers and away from the others
            row = torch.arange(rows, device="cuda")
            chosen = torch.searchsorted(s["end"].long(), row, right=True) % 2 == 0
            apart = torch.where(chosen, -0.05, 0.05) + 0.3 * torch.randn(rows, generator=g, device="cuda")
            s["ref"] = logp + apart
    return s


def run(s):
    if own:
        return _OWN[s["case"]["kind"]](s)
    return _PLAIN[s["case"]["kind"]](s)


# ------------------------------------------------------------------ the library's calls
def _scratch(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def _own_embed(s):
    from paper_2504_13850_amd import api as A

    case, stream, table = s["case"], torch.cuda.current_stream(), s["table"]
    out, dtable = torch.empty_like(s["dout"]), torch.empty_like(table)
    A.fo_embed_fwd(s["tokens"], table, out, scale=case["scale"], stream=stream)
    ws = _scratch(A.fo_embed_workspace(case["rows"], case["cols"], case["vocab"]))
    A.fo_embed_bwd(s["tokens"], s["dout"], dtable, scale=case["scale"], workspace=ws, stream=stream)
    return {"out": out, "dtable": dtable}


def _own_norm(s):
    from paper_2504_13850_amd import api as A

    x, w, stream = s["x"], s["w"], torch.cuda.current_stream()
    h = torch.empty_like(x) if s["case"]["residual"] else None
    y, rstd = torch.empty_like(x), torch.empty(len(x), device="cuda")
    A.fo_rmsnorm_fwd(x, w, y, rstd, EPS, residual=s["residual"], h=h, stream=stream)
    dx, dw, ws = torch.empty_like(x), torch.empty_like(w), _scratch(A.fo_rmsnorm_workspace(*x.shape))
    A.fo_rmsnorm_bwd(s["dy"], x if h is None else h, w, rstd, dx, dw, dres=s["dres"], workspace=ws, stream=stream)
    return {"y": y, "dx": dx, "dw": dw, **({} if h is None else {"h": h})}


def _own_norm8(s):
    from paper_2504_13850_amd import api as A

    x, stream = s["x"], torch.cuda.current_stream()
    q, scale = torch.empty(x.shape, dtype=F8, device="cuda"), torch.empty(len(x), device="cuda")
    if s["case"]["kind"] == "quant8":
        A.fo_quant_f8(x, q, scale, stream=stream)
        return {"q": q, "scale": scale}
    h = torch.empty_like(x) if s["case"]["residual"] else None
    A.fo_rmsnorm_f8(x, s["w"], q, scale, EPS, residual=s["residual"], h=h, stream=stream)
    return {"q": q, "scale": scale, **({} if h is None else {"h": h})}


def _own_gemm8(s):
    from paper_2504_13850_amd import api as A

    case = s["case"]
    c = torch.empty((case["m"], case["n"]), dtype=DT[case["dtype"]], device="cuda")
    ws = _scratch(A.fo_gemm_f8_workspace(case["m"], case["n"], case["k"]))
    A.fo_gemm_f8(s["a"], s["a_scale"], s["b"], s["b_scale"], c, workspace=ws, stream=torch.cuda.current_stream())
    return c


def _own_logp(s):
    from paper_2504_13850_amd import api as A

    case, logits, stream = s["case"], s["logits"], torch.cuda.current_stream()
    ws = _scratch(A.fo_logp_workspace(*logits.shape))
    logp = torch.empty(len(logits), device="cuda")
    if not case["train"]:
        A.fo_logp_fwd(logits, s["targets"], logp, scale=case["scale"], workspace=ws, stream=stream)
        return logp
    dlogits = torch.empty_like(logits)
    A.fo_xent(logits, s["targets"], s["weight"], logp, dlogits, scale=case["scale"], workspace=ws, stream=stream)
    return {"loss": logp, "dlogits": dlogits}


def _own_pref(s, logp=None, dlogp=None):
    from paper_2504_13850_amd import api as A

    case = s["case"]
    logp = s["logp"] if logp is None else logp
    loss, reward = torch.empty(case["pairs"], device="cuda"), torch.empty(2 * case["pairs"], device="cuda")
    dlogp = torch.empty_like(logp)
    A.fo_pref_loss(logp, s["ref"], s["begin"], s["end"], loss, reward, dlogp, beta=case["beta"], smooth=case["smooth"],
                   mean=case["mean"], dloss=1.0 / case["pairs"], stream=torch.cuda.current_stream())
    return {"loss": loss, "reward": reward, "dlogp": dlogp}


def _own_step(s):
    from paper_2504_13850_amd import api as A

    logits, stream = s["logits"], torch.cuda.current_stream()
    ws = _scratch(A.fo_logp_workspace(*logits.shape))
    logp, lse = torch.empty(len(logits), device="cuda"), torch.empty(len(logits), device="cuda")
    A.fo_logp_fwd(logits, s["targets"], logp, lse, workspace=ws, stream=stream)
    got = _own_pref(s, logp)
    dlogits = torch.empty_like(logits)
    A.fo_logp_bwd(logits, s["targets"], logp, lse, got["dlogp"], dlogits, stream=stream)
    return {"logp": logp, "loss": got["loss"], "reward": got["reward"], "dlogits": dlogits}


_OWN = {"embed": _own_embed, "norm": _own_norm, "norm8": _own_norm8, "quant8": _own_norm8, "gemm8": _own_gemm8,
        "logp": _own_logp, "pref": _own_pref, "step": _own_step}


# ------------------------------------------------------------------ plain torch, 32 bits
def _plain_embed(s):
    case, table = s["case"], s["table"]
    tok = s["tokens"].long()
    there = (tok >= 0) & (tok < case["vocab"])
    row, keep = torch.where(there, tok, 0), there[:, None].float() * case["scale"]
    out = (table[row].float() * keep).to(table.dtype)
    grad = torch.zeros(table.shape, dtype=torch.float32, device="cuda")
    grad.index_add_(0, row, s["dout"].float() * keep)
    return {"out": out, "dtable": grad.to(table.dtype)}


def _normed(s):
    """h, its reciprocal root mean square and the norm, in 32 bits."""
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    r = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    return h, r, h * r * s["w"].float()


def _plain_norm(s):
    dt = s["x"].dtype
    h, r, y = _normed(s)
    dy = s["dy"].float()
    g = dy * s["w"].float()
    dx = r * (g - h * (r * r * (g * h).mean(1, keepdim=True)))
    if s["dres"] is not None:
        dx = dx + s["dres"].float()
    got = {"y": y.to(dt), "dx": dx.to(dt), "dw": (dy * h * r).sum(0).to(dt)}
    return {**got, "h": h.to(dt)} if s["case"]["residual"] else got


def _plain_norm8(s):
    if s["case"]["kind"] == "quant8":
        h = y = s["x"].float()
    else:
        h, _, y = _normed(s)
    top = y.abs().amax(1)
    got = {"q": (y * (F8_MAX / top)[:, None]).clamp(-F8_MAX, F8_MAX).to(F8), "scale": top / F8_MAX}
    return {**got, "h": h.to(s["x"].dtype)} if s["case"]["residual"] else got


def _plain_gemm8(s):
    c = s["a"].float() @ s["b"].float().t()
    return (c * s["a_scale"][:, None] * s["b_scale"]).to(DT[s["case"]["dtype"]])


def _softmax_parts(s, scale):
    """The log probabilities of the targets (0 where there is none), and the softmax with the targets' places as
    minus the rest of the row: the gradient of minus logp.  The rest's sum is kept apart, since 1 - p loses all but
    a few bits where p is near 1; its logarithm is taken in 64 bits, since the preference loss adds up what logp is off
    by over whole answers."""
    z, t = s["logits"].float() * scale, s["targets"].long()
    there = (t >= 0) & (t < z.shape[1])
    t = torch.where(there, t, 0)[:, None]
    z = z - z.amax(1, keepdim=True)
    e = torch.exp(z)
    own_e, own_z = e.gather(1, t), z.gather(1, t)
    rest = e.scatter(1, t, 0.0).sum(1, keepdim=True).double()
    total = rest + own_e
    logp = torch.where(own_z == 0, -torch.log1p(rest / own_e), own_z - torch.log(total)).float()
    p = e / total.float()
    p.scatter_(1, t, (-rest / total).float())
    return torch.where(there, logp[:, 0], 0.0), p * there[:, None]


def _plain_logp(s):
    case = s["case"]
    logp, p = _softmax_parts(s, case["scale"])
    if not case["train"]:
        return logp
    return {"loss": -logp, "dlogits": (p * (s["weight"] * case["scale"])[:, None]).to(s["logits"].dtype)}


def _plain_pref(s, logp=None):
    """Sums over the answers in 64 bits: they are long, and the chosen's and the rejected's nearly cancel."""
    case = s["case"]
    logp = s["logp"] if logp is None else logp
    n = (s["end"] - s["begin"]).long()
    answer = torch.repeat_interleave(torch.arange(2 * case["pairs"], device="cuda"), n, output_size=len(logp))
    each = case["beta"] / n.clamp_min(1).double() if case["mean"] else torch.full(n.shape, case["beta"], device="cuda",
                                                                                  dtype=torch.float64)
    sums = torch.zeros(2 * case["pairs"], dtype=torch.float64, device="cuda")
    reward = sums.index_add(0, answer, logp.double() - s["ref"].double()) * each
    d = reward[0::2] - reward[1::2]
    soft = lambda x: x.clamp_min(0) + torch.log1p(torch.exp(-x.abs()))  # noqa: E731
    eps = case["smooth"]
    loss = (1 - eps) * soft(-d) + eps * soft(d)
    slope = (eps / (1 + torch.exp(-d)) - (1 - eps) / (1 + torch.exp(d))) / case["pairs"]
    dlogp = (torch.stack([slope, -slope], 1).flatten() * each)[answer]
    return {"loss": loss.float(), "reward": reward.float(), "dlogp": dlogp.float()}


def _plain_step(s):
    logp, p = _softmax_parts(s, 1.0)
    got = _plain_pref(s, logp)
    return {"logp": logp, "loss": got["loss"], "reward": got["reward"],
            "dlogits": (-p * got["dlogp"][:, None]).to(s["logits"].dtype)}


_PLAIN = {"embed": _plain_embed, "norm": _plain_norm, "norm8": _plain_norm8, "quant8": _plain_norm8,
          "gemm8": _plain_gemm8, "logp": _plain_logp, "pref": _plain_pref, "step": _plain_step}


# ------------------------------------------------------------------ the definitions, 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[case["kind"]](case, s)


def _exact_embed(case, s):
    table, tok = s["table"], s["tokens"].long()
    rows = torch.nonzero((tok >= 0) & (tok < case["vocab"]))[:, 0]
    out = torch.zeros(s["dout"].shape, dtype=torch.float64, device="cuda")
    out[rows] = table[tok[rows]].double() * case["scale"]
    grad = torch.zeros(table.shape, dtype=torch.float64, device="cuda")
    grad.index_put_((tok[rows],), s["dout"][rows].double() * case["scale"], accumulate=True)
    return {"out": out, "dtable": grad}


def _exact_norm(case, s):
    x = s["x"].double()
    h = x + s["residual"].double() if case["residual"] else x
    w, c = s["w"].double(), case["cols"]
    rms = ((h * h).sum(1, keepdim=True) / c + EPS).sqrt()
    unit = h / rms
    y = unit * w
    if case["kind"] == "norm8":
        top = y.abs().max(1).values
        return {"q": y / top[:, None] * F8_MAX, "scale": top / F8_MAX, **({"h": h} if case["residual"] else {})}
    dy = s["dy"].double()
    du = dy * w
    dx = (du - unit * ((du * unit).sum(1, keepdim=True) / c)) / rms
    if case["residual"]:
        dx += s["dres"].double()
    return {"y": y, "dx": dx, "dw": (dy * unit).sum(0), **({"h": h} if case["residual"] else {})}


def _exact_quant8(case, s):
    x = s["x"].double()
    top = x.abs().max(1).values
    return {"q": x / top[:, None] * F8_MAX, "scale": top / F8_MAX}


def _exact_gemm8(case, s):
    a, b = (s[n].float().double() * s[n + "_scale"].double()[:, None] for n in "ab")
    return a @ b.T


def _exact_rows(case, s, scale, weight):
    """Block by block: log probabilities, and `weight` (a function of the rows and their log probabilities) times the
    gradient of minus their sum; no gradient where weight is None."""
    logits, targets, v = s["logits"], s["targets"].long(), case["vocab"]
    logp = torch.zeros(len(logits), dtype=torch.float64, device="cuda")
    for r0 in range(0, len(logits), 1024):
        t = targets[r0:r0 + 1024]
        ok = torch.nonzero((t >= 0) & (t < v))[:, 0]
        full = torch.log_softmax(logits[r0:r0 + 1024].double()[ok] * scale, 1)
        logp[r0 + ok] = full[torch.arange(len(ok), device="cuda"), t[ok]]
    if weight is None:
        return logp, None
    by = weight(logp)
    grad = torch.zeros(logits.shape, dtype=torch.float64, device="cuda")
    for r0 in range(0, len(logits), 1024):
        t = targets[r0:r0 + 1024]
        ok = torch.nonzero((t >= 0) & (t < v))[:, 0]
        p = torch.softmax(logits[r0:r0 + 1024].double()[ok] * scale, 1)
        p[torch.arange(len(ok), device="cuda"), t[ok]] -= 1
        grad[r0 + ok] = p * by[r0 + ok][:, None] * scale
    return logp, grad


def _exact_logp(case, s):
    if not case["train"]:
        return _exact_rows(case, s, case["scale"], None)[0]
    logp, grad = _exact_rows(case, s, case["scale"], lambda _: s["weight"].double())
    return {"loss": -logp, "dlogits": grad}


def _exact_loss(case, s, logp):
    """Pair by pair on the host."""
    diff = (logp.double() - s["ref"].double()).cpu().numpy()
    spans = list(zip(s["begin"].tolist(), s["end"].tolist()))
    loss, reward, dlogp = np.zeros(case["pairs"]), np.zeros(2 * case["pairs"]), np.zeros(len(diff))
    for i in range(case["pairs"]):
        by = []
        for q in (2 * i, 2 * i + 1):
            lo, hi = spans[q]
            by.append(case["beta"] / (max(hi - lo, 1) if case["mean"] else 1))
            reward[q] = by[-1] * diff[lo:hi].sum()
        d, eps = reward[2 * i] - reward[2 * i + 1], case["smooth"]
        loss[i] = (1 - eps) * np.logaddexp(0, -d) + eps * np.logaddexp(0, d)
        slope = (eps * np.exp(-np.logaddexp(0, -d)) - (1 - eps) * np.exp(-np.logaddexp(0, d))) / case["pairs"]
        for q, sign in ((2 * i, 1.0), (2 * i + 1, -1.0)):
            dlogp[spans[q][0]:spans[q][1]] = sign * slope * by[q - 2 * i]
    return {n: torch.from_numpy(x).cuda() for n, x in (("loss", loss), ("reward", reward), ("dlogp", dlogp))}


def _exact_pref(case, s):
    return _exact_loss(case, s, s["logp"])


def _exact_step(case, s):
    got = {}

    def weight(logp):
        got.update(_exact_loss(case, s, logp))
        return -got.pop("dlogp")

    logp, grad = _exact_rows(case, s, 1.0, weight)
    return {"logp": logp, "dlogits": grad, **got}


_EXACT = {"embed": _exact_embed, "norm": _exact_norm, "norm8": _exact_norm, "quant8": _exact_quant8,
          "gemm8": _exact_gemm8, "logp": _exact_logp, "pref": _exact_pref, "step": _exact_step}

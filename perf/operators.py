"""The transformer operators beside the training steps, as cases to time and to check.

Three kinds of work, each through the public binding (paper_2504_13850_amd.api):

  train    masked attention on packed sequences, forward and backward: causal or
           prefix masks, scores capped by a tanh, a learned bias by distance
           bucket with its gradient, dropout of the probabilities
  infer    the same attention forward only; "one": one new token per sequence
           against a cache of earlier keys and values
  drop     dropout with bias and residual, forward, or forward and backward; the
           mask comes from a counter-based generator and is never stored

``own`` False computes them in plain torch at 32 bits, True calls the library.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    attn = {"kind": "train", "dtype": "bf16", "batch": 32, "heads": 12, "kv_heads": 12, "dim": 64, "min_len": 32,
            "max_len": 128, "lens_seed": 1, "mask": "full", "cap": 0.0, "buckets": 0, "radius": 0, "p": 0.0}
    drop = {"kind": "drop", "dtype": "bf16", "rows": 4096, "cols": 768, "p": 0.1, "bias": True, "residual": True,
            "train": True}
    return [
        # the encoder block of the BERT-shaped server network: 32 ragged sequences, learned bias, dropout
        dict(attn, name="train_bert_b32", buckets=32, radius=128, p=0.1),
        # the paper's transformers, fp32: 5 heads of width 20 on short sentences, 50 of width 2 on reviews
        dict(attn, name="train_tf6_b16", dtype="f32", batch=16, heads=5, kv_heads=5, dim=20, min_len=4, max_len=64,
             buckets=16, radius=32, p=0.1),
        dict(attn, name="train_tf12_b16", dtype="f32", batch=16, heads=50, kv_heads=50, dim=2, min_len=16,
             max_len=256, cap=30.0),
        # a causal language model on four packed documents of uneven length, grouped key heads, capped scores
        dict(attn, name="train_docs_4k", batch=4, heads=16, kv_heads=4, dim=128, min_len=500, max_len=4096,
             mask="causal", cap=50.0),
        # a prefix language model at middle length with the learned bias
        dict(attn, name="train_prefix_1k", batch=6, heads=12, kv_heads=4, dim=64, min_len=700, max_len=1023,
             mask="prefix", buckets=32, radius=128),
        # evaluation of a long causal batch
        dict(attn, name="infer_docs_8k", kind="infer", batch=2, heads=32, kv_heads=8, dim=128, min_len=5000,
             max_len=8191, mask="causal"),
        # single tokens: the shortest call there is, and a long cache shared by groups of four heads
        dict(attn, name="one_short", kind="one", batch=4, max_len=100, min_len=1, buckets=32, radius=64),
        dict(attn, name="one_cache_16k", kind="one", batch=16, heads=32, kv_heads=8, dim=128, min_len=6000,
             max_len=16384, cap=50.0, buckets=32, radius=128),
        # dropout between sublayers: the fp32 transformer's rows, BERT's, and a large forward pass
        dict(drop, name="drop_tf6", dtype="f32", rows=1024, cols=100, p=0.2),
        dict(drop, name="drop_bert", rows=4096, cols=768),
        dict(drop, name="drop_64k", rows=65536, cols=768, train=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {"flops": 0.0, "bytes": 0.0}
    for c in listed():
        most = {k: max(v, work(c)[k]) for k, v in most.items()}
    kind = rng.choice(["train", "train", "infer", "one", "drop"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "drop":
        case = {"kind": kind, "dtype": dtype, "rows": _log_int(rng, 1, 65536), "cols": _log_int(rng, 8, 2304),
                "p": rng.choice([0.05, 0.1, 0.25, 0.5]), "bias": rng.random() < 0.7, "residual": rng.random() < 0.7,
                "train": rng.random() < 0.6}
        while work(case)["bytes"] > most["bytes"]:
            case["rows"] = max(1, case["rows"] // 2)
        return case
    kv = rng.choice([1, 2, 4, 5, 8, 12])
    top, scores = {"train": (4096, 1 << 30), "infer": (8192, 1 << 32), "one": (16384, 1 << 32)}[kind]
    bias = rng.random() < 0.5
    hi = _log_int(rng, 2 if bias else 1, top)  # a lone key takes all the weight: the bias has no gradient
    case = {"kind": kind, "dtype": dtype, "batch": _log_int(rng, 1, 32), "heads": kv * rng.choice([1, 1, 2, 3, 4]),
            "kv_heads": kv, "dim": rng.choice([2, 20, 32, 48, 64, 64, 77, 80, 100, 128, 128]),
            "min_len": max(1, int(hi * rng.uniform(0.1, 1.0))), "max_len": hi, "lens_seed": rng.randint(1, 1000),
            "mask": "full" if kind == "one" else rng.choice(["full", "causal", "prefix"]),
            "cap": rng.choice([0.0, 0.0, 20.0, 50.0]), "buckets": rng.choice([16, 32]) if bias else 0,
            "radius": rng.choice([32, 128, 512]) if bias else 0,
            "p": rng.choice([0.0, 0.1, 0.2]) if kind == "train" else 0.0}
    queries = lambda c: 1 if kind == "one" else c["max_len"]  # noqa: E731
    while (work(case)["flops"] * (4 if dtype == "f32" else 1) > most["flops"] or work(case)["bytes"] > most["bytes"]
           or case["batch"] * case["heads"] * queries(case) * case["max_len"] > scores):  # the plain form holds them
        if case["batch"] > 1:
            case["batch"] //= 2
        else:
            case["max_len"] = max(1, case["max_len"] // 2)
            case["min_len"] = min(case["min_len"], case["max_len"])
    return case


# ------------------------------------------------------------------ what a case holds
def _lens(case):
    """The keys of each sequence, the same for every seed; the first is the longest."""
    r = random.Random(case["lens_seed"])
    lens = [r.randint(case["min_len"], case["max_len"]) for _ in range(case["batch"])]
    lens[0] = case["max_len"]
    return lens


def _prefix(case, lens):
    return [n // 3 for n in lens] if case["mask"] == "prefix" else None


def _pairs(case):
    """(query, key) pairs that see each other, over the batch, for one head."""
    lens = _lens(case)
    if case["kind"] == "one":
        return float(sum(lens))
    if case["mask"] == "full":
        return float(sum(n * n for n in lens))
    pre = _prefix(case, lens) or [0] * len(lens)
    return float(sum(n * (n + 1) // 2 + m * (m - 1) // 2 for n, m in zip(lens, pre)))


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "drop":
        n = case["rows"] * case["cols"]
        passes = 2 + case["residual"] + (2 if case["train"] else 0)  # x (and residual) in, y out; dy in, dx out
        return {"bytes": float(passes * n * size), "flops": 0.0}
    h, kv, d, t = case["heads"], case["kv_heads"], case["dim"], sum(_lens(case))
    tq = case["batch"] if case["kind"] == "one" else t
    once = (2 * tq * h + 2 * t * kv) * d * size  # q in, out out, k and v in
    p = _pairs(case) * h * d
    if case["kind"] != "train":
        return {"bytes": float(once), "flops": 4.0 * p}
    return {"bytes": float(2 * once + tq * h * d * size), "flops": 14.0 * p}  # the backward reads out's gradient too


def _buckets(n_buckets, radius, causal):
    """The bucket of each distance key - query in [-radius, radius]: near distances one each, far ones in
    logarithmic steps; half of the buckets for each direction, or all of them for earlier keys."""
    half = n_buckets if causal else n_buckets // 2
    near = half // 2
    out = []
    for n in range(-radius, radius + 1):
        a = max(-n, 0) if causal else abs(n)
        b = a if a < near else min(half - 1, near + int(math.log(a / near) / math.log(radius / near) * (half - near) + 1e-9))
        out.append(b + (half if n > 0 and not causal else 0))
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = DT[case["dtype"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)

    s = {"case": case, "key": random.Random(seed).getrandbits(64), "offset": random.Random(seed + 1).getrandbits(32)}
    if case["kind"] == "drop":
        r, c = case["rows"], case["cols"]
        s.update(x=normal(r, c), bias=normal(c, scale=0.1) if case["bias"] else None,
                 residual=normal(r, c) if case["residual"] else None, dy=normal(r, c) if case["train"] else None)
        return s
    lens, h, kv, d = _lens(case), case["heads"], case["kv_heads"], case["dim"]
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    if case["kind"] == "one":  # a cache of max_len rows for each sequence, filled up to its length
        b, room = case["batch"], case["max_len"]
        s.update(q=normal(b, h, d), k=normal(b * room, kv, d), v=normal(b * room, kv, d), max_q=1,
                 q_begin=on(range(b)), q_end=on(range(1, b + 1)), k_begin=on([i * room for i in range(b)]),
                 k_end=on([i * room + n for i, n in enumerate(lens)]))
    else:  # the fused projection's rows, as a step has them: q, k and v are columns of one matrix
        at = [0]
        for n in lens:
            at.append(at[-1] + n)
        qkv = normal(at[-1], (h + 2 * kv) * d)
        cut = lambda i, n: qkv[:, i * d:(i + n) * d].unflatten(1, (n, d))  # noqa: E731
        s.update(q=cut(0, h), k=cut(h, kv), v=cut(h + kv, kv), max_q=max(lens), q_begin=on(at[:-1]), q_end=on(at[1:]))
        s.update(k_begin=s["q_begin"], k_end=s["q_end"])
    pre = _prefix(case, lens)
    s.update(max_k=max(lens), prefix=on(pre) if pre else None, table=None, bucket=None,
             dout=normal(*s["q"].shape) if case["kind"] == "train" else None)
    if case["buckets"]:
        s.update(table=normal(case["buckets"], h, scale=0.5),
                 bucket=on(_buckets(case["buckets"], case["radius"], case["mask"] == "causal")))
    return s


def run(s):
    if s["case"]["kind"] == "drop":
        return _own_drop(s) if own else _plain_drop(s)
    return _own_attention(s) if own else _plain_attention(s)


# ------------------------------------------------------------------ the library's calls
def _own_attention(s):
    from paper_2504_13850_amd import api as A

    case, q, k, v = s["case"], s["q"], s["k"], s["v"]
    train = case["kind"] == "train"
    stream = torch.cuda.current_stream()
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    a = A.make_attn(q, k, v, out, s["q_begin"], s["q_end"], s["k_begin"], s["k_end"], s["max_q"], s["max_k"],
                    cap=case["cap"], mask={"full": A.FO_ATTN_FULL, "causal": A.FO_ATTN_CAUSAL,
                                           "prefix": A.FO_ATTN_PREFIX}[case["mask"]],
                    prefix=s["prefix"], table=s["table"], bucket=s["bucket"], p=case["p"], seed=s["key"],
                    offset=s["offset"])
    lse = torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=q.device) if train else None
    n = A.fo_attn_workspace(a, train)
    ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    A.fo_attn_fwd(a, q, k, v, out, lse, ws, stream=stream)
    if not train:
        return out
    h, kv, d = q.shape[1], k.shape[1], q.shape[2]
    dqkv = torch.empty((q.shape[0], (h + 2 * kv) * d), dtype=q.dtype, device=q.device)
    dq, dk, dv = (t.unflatten(1, (-1, d)) for t in dqkv.split((h * d, kv * d, kv * d), 1))
    dtable = None if s["table"] is None else torch.empty_like(s["table"])
    A.fo_attn_bwd(a, q, k, v, out, lse, s["dout"], dq, dk, dv, dtable, ws, stream=stream)
    return {"out": out, "dqkv": dqkv, **({} if dtable is None else {"dtable": dtable})}


def _own_drop(s):
    from paper_2504_13850_amd import api as A

    case, x, stream = s["case"], s["x"], torch.cuda.current_stream()
    y = torch.empty_like(x)
    A.fo_dropout_fwd(x, y, case["p"], s["key"], s["offset"], bias=s["bias"], residual=s["residual"], stream=stream)
    if not case["train"]:
        return y
    dx, dbias, ws = torch.empty_like(x), None, None
    if case["bias"]:
        dbias = torch.empty_like(s["bias"])
        ws = torch.empty(A.fo_dropout_workspace(case["rows"], case["cols"]), dtype=torch.uint8, device=x.device)
    A.fo_dropout_bwd(s["dy"], dx, case["p"], s["key"], s["offset"], dbias=dbias, workspace=ws, stream=stream)
    return {"y": y, "dx": dx, **({} if dbias is None else {"dbias": dbias})}


# ------------------------------------------------------------------ plain torch, 32 bits
LOW = 0xFFFFFFFF


def _round(c, key):
    """One round of the generator on four counter words (int64 tensors below 2^32)."""
    a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57  # products mod 2^64
    return ((b >> 32) & LOW) ^ c[1] ^ key[0], b & LOW, ((a >> 32) & LOW) ^ c[3] ^ key[1], a & LOW


def _halves(c, seed):
    """Philox 4x32 with seven rounds (Salmon et al., 2011): the eight 16-bit halves of the output, low first."""
    key, k0, k1 = (seed & LOW, seed >> 32), seed & LOW, seed >> 32
    for r in range(7):
        key = ((k0 + r * 0x9E3779B9) & LOW, (k1 + r * 0xBB67AE85) & LOW)
        c = _round(c, key)
    return torch.stack([(w >> sh) & 0xFFFF for w in c for sh in (0, 16)], -1)


def _threshold(p):
    return int(math.floor(p * 65536 + 0.5))


def _attention_keep(case, b, lq, lk, seed, offset, dev):
    """1 / (1 - p) where a probability is kept, 0 where it is dropped: [batch, heads, lq, lk]."""
    ar = lambda n: torch.arange(n, device=dev, dtype=torch.int64)  # noqa: E731
    h, blocks = case["heads"], (lk + 15) // 16
    seq = (ar(b)[:, None] * h + ar(h)).view(b, h, 1, 1)
    c = torch.broadcast_tensors(ar(2 * blocks), ar(lq)[:, None], seq, torch.full((), offset, device=dev))
    half = _halves(c, seed).view(b, h, lq, blocks, 2, 2, 4)  # block of 16 keys, key bit 2, key bit 3, key bits 0-1
    half = half.transpose(4, 5).reshape(b, h, lq, blocks * 16)[..., :lk]
    t = _threshold(case["p"])
    return (half >= t).float() * (65536.0 / (65536 - t))


def _plain_attention(s):
    case, dev = s["case"], s["q"].device
    h, kv, d, b = case["heads"], case["kv_heads"], case["dim"], case["batch"]
    ar = lambda n: torch.arange(n, device=dev, dtype=torch.int64)  # noqa: E731

    def rows(begin, end, most):  # each sequence's rows, and which of them there are
        at = begin.long()[:, None] + ar(most)
        ok = at < end.long()[:, None]
        return torch.where(ok, at, 0), ok

    def padded(x, at, ok):  # [batch, heads, rows, dim]
        return (x.float()[at] * ok[:, :, None, None]).transpose(1, 2).contiguous()

    lq, lk = s["max_q"], s["max_k"]
    qi, qok = rows(s["q_begin"], s["q_end"], lq)
    ki, kok = rows(s["k_begin"], s["k_end"], lk)
    group = ar(h) // (h // kv)
    q, k, v = padded(s["q"], qi, qok), padded(s["k"], ki, kok)[:, group], padded(s["v"], ki, kok)[:, group]
    nq, nk = (s["q_end"] - s["q_begin"]).long(), (s["k_end"] - s["k_begin"]).long()
    dist = ar(lk) - ar(lq)[:, None] - (nk - nq)[:, None, None]  # the last query stands at the last key
    seen = kok[:, None, :] & qok[:, :, None]
    if case["mask"] != "full":
        late = dist <= 0
        if s["prefix"] is not None:
            late = late | (ar(lk) < s["prefix"].long()[:, None])[:, None, :]
        seen = seen & late
    scale, cap = d ** -0.5, case["cap"]
    u = q @ k.transpose(2, 3).contiguous() * scale
    if cap:
        t = torch.tanh(u / cap)
        u = cap * t
    if s["table"] is not None:
        r = case["radius"]
        of = s["bucket"].long()[dist.clamp(-r, r) + r]
        u = u + s["table"].float()[of].permute(0, 3, 1, 2)
    u = u.masked_fill(~seen[:, None], -math.inf)
    top = u.amax(-1, keepdim=True)
    e = torch.exp(u - torch.where(top == -math.inf, 0.0, top))
    p = e / e.sum(-1, keepdim=True).clamp_min(1e-37)
    keep = _attention_keep(case, b, lq, lk, s["key"], s["offset"], dev) if case["p"] else None
    pk = p if keep is None else p * keep

    def packed(x, ok):  # back to the rows in order
        return x.transpose(1, 2)[ok]

    out = packed(pk @ v, qok).to(s["q"].dtype)
    if case["kind"] != "train":
        return out
    do = padded(s["dout"], qi, qok)
    shared = lambda x: x.view(b, kv, h // kv, *x.shape[2:]).sum(2)  # noqa: E731
    dv = shared(pk.transpose(2, 3).contiguous() @ do)
    dp = do @ v.transpose(2, 3).contiguous()
    if keep is not None:
        dp = dp * keep
    du = p * (dp - (p * dp).sum(-1, keepdim=True))
    ds = (du * (1 - t * t) if cap else du) * scale
    dk = shared(ds.transpose(2, 3).contiguous() @ q)
    parts = [packed(x, ok).flatten(1) for x, ok in ((ds @ k, qok), (dk, kok), (dv, kok))]
    got = {"out": out, "dqkv": torch.cat(parts, 1).to(s["q"].dtype)}
    if s["table"] is not None:
        # sums along the diagonals: rows in reverse order, one column longer each, so that a distance is a column
        wide = torch.nn.functional.pad(du.sum(0).flip(1), (0, lq)).flatten(1)[:, :-lq].view(h, lq, lk + lq - 1)
        on = (s["bucket"].long()[(ar(lk + lq - 1) - (lq - 1)).clamp(-r, r) + r][:, None] == ar(case["buckets"])).float()
        got["dtable"] = (wide.sum(1) @ on).t().to(s["q"].dtype)
    return got


def _plain_drop(s):
    case, x = s["case"], s["x"]
    rows, cols = x.shape
    calls = (cols + 7) // 8
    n = torch.arange(rows * calls, device=x.device, dtype=torch.int64)
    zero = torch.zeros((), dtype=torch.int64, device=x.device)
    half = _halves((n & LOW, n >> 32, zero, zero + s["offset"]), s["key"])
    t = _threshold(case["p"])
    keep = (half >= t).view(rows, calls * 8)[:, :cols].float() * (65536.0 / (65536 - t))
    y = x.float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = y * keep
    if s["residual"] is not None:
        y = y + s["residual"].float()
    y = y.to(x.dtype)
    if not case["train"]:
        return y
    dx = s["dy"].float() * keep
    got = {"y": y, "dx": dx.to(x.dtype)}
    if s["bias"] is not None:
        got["dbias"] = dx.sum(0).to(x.dtype)
    return got


# ------------------------------------------------------------------ the definitions, 64 bits
def _philox(c0, c1, c2, c3, seed):
    """The generator on numpy's unsigned words: [..., 8] halves."""
    m0, m1, low = np.uint64(0xD2511F53), np.uint64(0xCD9E8D57), np.uint64(LOW)
    sh = np.uint64(32)
    c = [np.asarray(v, np.uint64) for v in (c0, c1, c2, c3)]
    for r in range(7):
        k0 = np.uint64(((seed & LOW) + r * 0x9E3779B9) & LOW)
        k1 = np.uint64(((seed >> 32) + r * 0xBB67AE85) & LOW)
        x, y = c[0] * m0, c[2] * m1
        c = [(y >> sh) ^ c[1] ^ k0, y & low, (x >> sh) ^ c[3] ^ k1, x & low]
    words = np.stack(np.broadcast_arrays(*c), -1).astype(np.uint32)
    return np.stack([words & 0xFFFF, words >> 16], -1).reshape(words.shape[:-1] + (8,))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "drop":
        if case["rows"] * case["cols"] > 1 << 26:
            return None
        return _exact_drop(case, s)
    if case["p"] and _pairs(case) * case["heads"] > 3e8:
        return None
    return _exact_attention(case, s)


def _exact_drop(case, s):
    rows, cols = case["rows"], case["cols"]
    calls = (cols + 7) // 8
    n = np.arange(rows * calls, dtype=np.uint64).reshape(rows, calls)
    half = _philox(n & np.uint64(LOW), n >> np.uint64(32), 0, s["offset"], s["key"]).reshape(rows, -1)[:, :cols]
    t = _threshold(case["p"])
    keep = torch.from_numpy((half >= t) / (1 - t / 65536)).cuda()
    y = (s["x"].double() + (0 if s["bias"] is None else s["bias"].double())) * keep
    if s["residual"] is not None:
        y = y + s["residual"].double()
    if not case["train"]:
        return y
    dx = keep * s["dy"].double()
    return {"y": y, "dx": dx, **({"dbias": dx.sum(0)} if case["bias"] else {})}


def _exact_attention(case, s):
    """Sequence by sequence and head by head."""
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    q, k, v = (s[n].double() for n in "qkv")
    train, r = case["kind"] == "train", case["radius"]
    out, dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dtable = torch.zeros((case["buckets"], h), dtype=torch.float64, device=q.device)
    thr = _threshold(case["p"])
    spans = list(zip(*(s[n].tolist() for n in ("q_begin", "q_end", "k_begin", "k_end"))))
    for b, (q0, q1, k0, k1) in enumerate(spans):
        lq, lk = q1 - q0, k1 - k0
        i = torch.arange(lq, device=q.device)[:, None] + (lk - lq)
        j = torch.arange(lk, device=q.device)[None]
        hide = torch.zeros((lq, lk), dtype=torch.bool, device=q.device)
        if case["mask"] != "full":
            hide = j > i
        if case["mask"] == "prefix":
            hide = hide & (j >= int(s["prefix"][b]))
        of = s["bucket"].long()[torch.clamp(j - i, -r, r) + r] if r else None
        for n in range(h):
            m = n // (h // kv)
            x, kk, vv = q[q0:q1, n], k[k0:k1, m], v[k0:k1, m]
            a = (x @ kk.T) / math.sqrt(d)
            c = case["cap"] * torch.tanh(a / case["cap"]) if case["cap"] else a
            z = c + s["table"].double()[:, n][of] if r else c
            p = torch.softmax(z.masked_fill(hide, -math.inf), 1)
            if case["p"]:
                key = np.arange(lk)
                call = 2 * (key // 16) + (key // 4) % 2
                half = _philox(np.arange(0, 2 * ((lk + 15) // 16))[None], np.arange(lq)[:, None], b * h + n,
                               s["offset"], s["key"])[:, call, key % 4 + 4 * ((key // 8) % 2)]
                keep = torch.from_numpy((half >= thr) / (1 - thr / 65536)).to(q.device)
            else:
                keep = 1.0
            out[q0:q1, n] = (p * keep) @ vv
            if not train:
                continue
            do = s["dout"][q0:q1, n].double()
            dv[k0:k1, m] += (p * keep).T @ do
            dp = (do @ vv.T) * keep
            dz = p * (dp - (p * dp).sum(1, keepdim=True))
            if r:
                dtable[:, n].index_add_(0, of.reshape(-1), dz.reshape(-1))
            if case["cap"]:
                dz = dz * (1 - (c / case["cap"]) ** 2)
            dq[q0:q1, n] = dz @ kk / math.sqrt(d)
            dk[k0:k1, m] += dz.T @ x / math.sqrt(d)
    if not train:
        return out
    got = {"out": out, "dqkv": torch.cat([t.flatten(1) for t in (dq, dk, dv)], 1)}
    return {**got, "dtable": dtable} if r else got

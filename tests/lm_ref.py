"""Plain 64-bit statements of a language model's operators around its attention (embedding, RMS norm, 8-bit rows and
their product, log probabilities, preference loss), each beside what its kernel's roundings may add up to: arrays of
the results and, under "...~", of the sums of absolute terms that an fp32 evaluation's error is proportional to."""
import numpy as np

F8_MAX, TINY = 448.0, 2.0 ** -100


def embed(tokens, table, scale):
    ok = (tokens >= 0) & (tokens < len(table))
    out = np.zeros((len(tokens), table.shape[1]))
    out[ok] = scale * table[tokens[ok]]
    return out


def embed_grad(tokens, dout, scale, vocab, old=None):
    """dtable and, per element, the sum of its terms' sizes and their number."""
    ok = (tokens >= 0) & (tokens < vocab)
    got, size, count = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1])), np.zeros((vocab, 1))
    np.add.at(got, tokens[ok], scale * dout[ok])
    np.add.at(size, tokens[ok], abs(scale * dout[ok]))
    np.add.at(count, tokens[ok], 1)
    if old is not None:
        got, size, count = got + old, size + abs(old), count + 1
    return got, size, count


def rmsnorm(x, res, w, eps):
    """h, rstd, y."""
    h = x if res is None else x + res
    mean = (h * h).mean(1, keepdims=True) + eps
    r = np.where(mean > 0, 1 / np.sqrt(np.where(mean > 0, mean, 1)), 0)
    return h, r[:, 0], h * r * (1 if w is None else w)


def rmsnorm_grad(dy, h, w, rstd, dres):
    """dx, dw and the sizes of their terms."""
    r, n = rstd[:, None], h.shape[1]
    g = dy if w is None else dy * w
    dx = r * (g - h * r * r * (g * h).sum(1, keepdims=True) / n)
    size = abs(r) * (abs(g) + abs(h) * r * r * abs(g * h).sum(1, keepdims=True) / n)
    if dres is not None:
        dx, size = dx + dres, size + abs(dres)
    return dx, (dy * h * r).sum(0), size, abs(dy * h * r).sum(0)


def f8_values():
    """What the 256 bytes stand for: sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7F and 0xFF are NaN."""
    v = np.zeros(256)
    for i in range(256):
        e, m = (i >> 3) & 15, i & 7
        v[i] = (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) * (-1 if i >> 7 else 1)
    v[[0x7F, 0xFF]] = np.nan
    return v


def f8_scale(y):
    """The rows' scales: largest over 448, 2^-100 in place of smaller ones, 0 for zeros."""
    top = abs(y).max(1)
    return np.where((top > 0) & (top < TINY), TINY, top) / F8_MAX


def gemm(a, sa, b, sb):
    """The product and the sum of its terms' sizes."""
    scale = (1 if sa is None else sa[:, None]) * (1 if sb is None else sb)
    return a @ b.T * scale, abs(a) @ abs(b).T * abs(scale)


def logp(logits, targets, scale):
    """logp, lse, probabilities, and z less its maximum; ignored rows hold 0, rows without any term -infinity."""
    z = scale * logits
    rows, v = z.shape
    there = (targets >= 0) & (targets < v)
    t = np.where(there, targets, 0)
    top = z.max(1)
    top = np.where(np.isfinite(top), top, 0)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.exp(z - top[:, None])
        rest = e.copy()
        rest[np.arange(rows), t] = 0
        rest, own = rest.sum(1), e[np.arange(rows), t]
        lp = np.where(own > 0.5, -np.log1p(rest / own), z[np.arange(rows), t] - top - np.log(rest + own))
        lse = top + np.log(rest + own)
        p = e / (rest + own)[:, None]
        miss = rest / (rest + own)  # 1 - p of the target
    none = (rest + own) == 0
    lp, lse = np.where(none, -np.inf, lp), np.where(none, -np.inf, lse)
    return np.where(there, lp, 0), np.where(there, lse, 0), p, miss, there, none


def logp_grad(logits, targets, scale, g):
    """The gradient of sum g logp, given the rows' g."""
    lp, lse, p, miss, there, none = logp(logits, targets, scale)
    d = -p
    d[np.arange(len(d)), np.where(there, targets, 0)] = miss
    d[~there | none] = 0
    return scale * np.where(there, g, 0)[:, None] * d


def pref(logp, ref, spans, beta, smooth, mean, dloss):
    """loss, reward, dlogp (NaN in rows of no answer), and d."""
    diff = logp if ref is None else logp - ref
    pairs = len(spans) // 2
    by = [beta / max(1, hi - lo) if mean else beta for lo, hi in spans]
    reward = np.array([b * diff[lo:hi].sum() for b, (lo, hi) in zip(by, spans)])
    d = reward[0::2] - reward[1::2]
    loss = (1 - smooth) * np.logaddexp(0, -d) + smooth * np.logaddexp(0, d)
    sig = lambda x: np.exp(-np.logaddexp(0, -x))  # noqa: E731
    slope = dloss * (smooth * sig(d) - (1 - smooth) * sig(-d))
    size = abs(dloss) * (smooth * sig(d) + (1 - smooth) * sig(-d))
    g, gs = np.full(len(diff), np.nan), np.full(len(diff), np.nan)
    for i in range(pairs):
        for q, sign in ((2 * i, 1), (2 * i + 1, -1)):
            lo, hi = spans[q]
            g[lo:hi], gs[lo:hi] = sign * slope[i] * by[q], size[i] * abs(by[q])
    return loss, reward, g, gs, d

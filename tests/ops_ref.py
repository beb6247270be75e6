"""Plain 64-bit statements of the transformer operators, for their tests.

Attention goes sequence by sequence and head by head over whole score
matrices; the dropout generator runs on numpy's unsigned words.  Beside each
result stands a scale for its error: the root of the summed squares of the
terms that the result adds up, without the cancellation between them.
"""
import numpy as np

LOW = np.uint64(0xFFFFFFFF)


def philox7(c0, c1, c2, c3, seed):
    """Philox 4x32 with seven rounds: [..., 4] words."""
    sh = np.uint64(32)
    c = [np.asarray(v, np.uint64) for v in (c0, c1, c2, c3)]
    for r in range(7):
        k0 = np.uint64(((seed & 0xFFFFFFFF) + r * 0x9E3779B9) & 0xFFFFFFFF)
        k1 = np.uint64(((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> sh) ^ c[1] ^ k0, b & LOW, (a >> sh) ^ c[3] ^ k1, a & LOW]
    return np.stack(np.broadcast_arrays(*c), -1).astype(np.uint32)


def halves(words):
    return np.stack([words & 0xFFFF, words >> 16], -1).reshape(words.shape[:-1] + (8,))


def threshold(p):
    return min(65535, int(np.floor(float(np.float32(p)) * 65536 + 0.5)))


def drop_matrix(rows, cols, p, seed, offset):
    t = threshold(p)
    calls = -(-cols // 8)
    n = np.arange(rows * calls, dtype=np.uint64)
    h = halves(philox7(n & LOW, n >> np.uint64(32), 0, offset, seed)).reshape(rows, calls * 8)[:, :cols]
    return (h >= t) / (1 - t / 65536)


def drop_scores(lq, lk, bh, p, seed, offset):
    t = threshold(p)
    j = np.arange(lk)
    h = halves(philox7((2 * (j // 16) + (j // 4) % 2)[None], np.arange(lq)[:, None], bh, offset, seed))
    pick = np.broadcast_to(j % 4 + 4 * ((j // 8) % 2), (lq, lk))
    return (np.take_along_axis(h, pick[..., None], -1)[..., 0] >= t) / (1 - t / 65536)


def attention(q, k, v, spans, mask, scale, cap=0.0, prefix=None, table=None, bucket=None, p=0.0, seed=0, offset=0,
              dout=None):
    """q [rows, heads, dim], k and v [rows, kv_heads, dim] (float64), spans (q0, q1, k0, k1) per sequence.  Returns a
    dict of (value, scale of its error); rows of no sequence are NaN."""
    H, KV, G = q.shape[1], k.shape[1], q.shape[1] // k.shape[1]
    names = ["out"] + ([] if dout is None else ["dq", "dk", "dv"])
    like = {"out": q, "dq": q, "dk": k, "dv": v}
    got = {n: [np.full(like[n].shape, np.nan), np.full(like[n].shape, np.nan)] for n in names}
    if table is not None and dout is not None:
        got["dtable"] = [np.zeros(table.shape), np.zeros(table.shape)]
    lse = np.full((H, q.shape[0]), np.nan)
    for b, (q0, q1, k0, k1) in enumerate(spans):
        lq, lk = q1 - q0, k1 - k0
        for n in names:
            lo, hi = (q0, q1) if n in ("out", "dq") else (k0, k1)
            for x in got[n]:
                x[lo:hi] = 0
        n = np.arange(lk)[None] - np.arange(lq)[:, None] - (lk - lq)
        seen = np.ones((lq, lk), bool)
        if mask:
            seen = n <= 0
        if mask == 2:
            seen = seen | (np.arange(lk)[None] < prefix[b])
        if table is not None:
            R = len(bucket) // 2
            of = np.clip(bucket[np.clip(n, -R, R) + R], 0, len(table) - 1)
        for h in range(H):
            m = h // G
            qq, kk, vv = q[q0:q1, h], k[k0:k1, m], v[k0:k1, m]
            c = scale * qq @ kk.T
            slope = np.ones_like(c)
            if cap:
                t = np.tanh(c / cap)
                c, slope = cap * t, 1 - t * t
            u = c
            if table is not None:
                bias = table[of, h]
                u = np.where(bias <= -1e30, -np.inf, u + bias)
            u = np.where(seen, u, -np.inf)
            top = u.max(1, keepdims=True) if lk else np.zeros((lq, 1))
            e = np.exp(u - np.where(np.isfinite(top), top, 0))
            l = e.sum(1, keepdims=True)
            P = e / np.where(l > 0, l, 1)
            with np.errstate(divide="ignore"):
                lse[h, q0:q1] = (np.log(l) + np.where(np.isfinite(top), top, 0))[:, 0]
            drop = drop_scores(lq, lk, b * H + h, p, seed, offset) if p else np.ones_like(P)
            Pd = P * drop
            got["out"][0][q0:q1, h] = Pd @ vv
            got["out"][1][q0:q1, h] = np.sqrt(Pd ** 2 @ vv ** 2)
            if dout is None:
                continue
            g = dout[q0:q1, h]
            dP = (g @ vv.T) * drop
            delta = (P * dP).sum(1, keepdims=True)
            dU = P * (dP - delta)
            A2 = P ** 2 * (((g ** 2 @ vv.T ** 2) * drop ** 2) + delta ** 2)  # squared terms of dU
            if table is not None:
                np.add.at(got["dtable"][0][:, h], of, dU)
                np.add.at(got["dtable"][1][:, h], of, A2)
            dS = dU * slope
            got["dq"][0][q0:q1, h] = scale * dS @ kk
            got["dq"][1][q0:q1, h] = abs(scale) * np.sqrt(A2 @ kk ** 2)
            got["dk"][0][k0:k1, m] += scale * dS.T @ qq
            got["dk"][1][k0:k1, m] += scale ** 2 * (A2.T @ qq ** 2)  # rooted below
            got["dv"][0][k0:k1, m] += Pd.T @ g
            got["dv"][1][k0:k1, m] += (Pd ** 2).T @ g ** 2
    for n in ("dk", "dv", "dtable"):
        if n in got:
            got[n][1] = np.sqrt(got[n][1])
    return {n: tuple(x) for n, x in got.items()}, lse

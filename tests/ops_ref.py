"""Plain implementations, in 64 bits, of the operators on the pool's contents, with bounds on what the library's arithmetic may
differ by.  Written from the definitions in include/kvswap.h; they share no code with the library.

Pools are numpy arrays [L, 2, N, B, H, D] of float64 (the values that the stored elements stand for, scales applied).
Bounds: u is the unit roundoff of the 16-bit type (2^-8 for bf16, 2^-11 for f16).  A score q.k of D products in 32 bits is off by at
most (D + 4) 2^-23 times the sum of the products' magnitudes; a softmax weight then by its own size times twice that and a few roundings,
its rounding to 16 bits for the product with V by u of itself, and the result is rounded once to the type.
"""
import numpy as np

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def csr(rows):
    off = np.zeros(len(rows) + 1, np.int32)
    off[1:] = np.cumsum([len(r) for r in rows])
    return off, (np.concatenate(rows) if off[-1] else np.zeros(0)).astype(np.int32)


def request_rows(pool_layer, table, length, B):
    """(2, length, H, D): keys and values of a request in order."""
    x = np.arange(length)
    return pool_layer[:, np.asarray(table, np.int64)[x // B], x % B]


def attention(pool_layer, tables, lens, q_lens, q, scale, io, B):
    """q [T, Hq, D] float64 -> (out, out bound, lse, lse bound, list of weights [H, length], list of their bounds)"""
    H, D = pool_layer.shape[3], pool_layer.shape[4]
    T, Hq = q.shape[:2]
    G = Hq // H
    u = U[io]
    out, tol = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, ltol = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    weights, wtol = [], []
    t = 0
    for table, length, new in zip(tables, lens, q_lens):
        kv = request_rows(pool_layer, table, length, B)
        w, wt = np.zeros((H, length)), np.zeros((H, length))
        for j in range(new):
            seen = length - new + j + 1 if length else 0
            for hq in range(Hq if seen > 0 else 0):
                h = hq // G
                k, v = kv[0, :seen, h], kv[1, :seen, h]
                with np.errstate(invalid="ignore", over="ignore"):
                    z = k @ q[t, hq] * scale
                    ds = ((D + 4) * 2.0 ** -23 * (np.abs(k) @ np.abs(q[t, hq])) * abs(scale)).max() + 2.0 ** -22 * np.abs(z).max() + 2.0 ** -20
                    m = z.max()
                    e = np.exp(z - m)
                    total = e.sum()
                    p = e / total
                    out[t, hq] = p @ v
                    spread = p @ np.abs(v)
                    tol[t, hq] = u * np.abs(out[t, hq]) + spread * (u + 2 * ds + (seen + 64) * 2.0 ** -23) + 1e-30
                    lse[t, hq] = m + np.log(total)
                    ltol[t, hq] = 2 * ds + 2.0 ** -22 * (1 + np.abs(lse[t, hq]))
                w[h, :seen] += p
                wt[h, :seen] += p * (4 * ds + 2.0 ** -20)
            t += 1
        weights.append(w)
        wtol.append(wt)
    return out, tol, lse, ltol, weights, wtol


def rotate(x, positions, freq_turns, magnitude, interleaved):
    """x [T, heads, D] float64; freq_turns [rot/2] in turns a position -> (turned, sum of the two products' magnitudes)"""
    rot = 2 * len(freq_turns)
    y, mag = x.copy(), np.abs(x)
    # turns modulo one, in integers of 2^-64: no position is too large
    word = np.round(np.asarray(freq_turns, np.longdouble) * np.longdouble(2) ** 64).astype(object)
    for t, p in enumerate(positions):
        ang = np.array([(int(w) * int(p)) % (1 << 64) / 2.0 ** 64 for w in word]) * 2 * np.pi
        c, s = np.cos(ang) * magnitude, np.sin(ang) * magnitude
        a_at = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
        b_at = a_at + 1 if interleaved else a_at + rot // 2
        a, b = x[t][:, a_at], x[t][:, b_at]
        y[t][:, a_at], y[t][:, b_at] = a * c - b * s, b * c + a * s
        mag[t][:, a_at] = mag[t][:, b_at] = (np.abs(a) + np.abs(b)) * abs(magnitude)
    return y, mag


def evict_kept(weights, length, keep, first, last):
    """Indices that stay of one head's row of weights."""
    if length <= keep:
        return np.arange(length)
    mid = np.arange(first, length - last)
    key = np.where(np.isnan(weights[mid]), -np.inf, weights[mid].astype(np.float64))
    nan = np.isnan(weights[mid])
    order = sorted(range(len(mid)), key=lambda i: (nan[i], -key[i], mid[i]))[:keep - first - last]
    return np.sort(np.concatenate([np.arange(first), mid[order], np.arange(length - last, length)])).astype(np.int64)

"""Plain implementations, in 64 bits, of the operators on drafted trees and of rotary positions with several axes.  Written from the definitions in
include/kvswap.h; they share no code with the library.  Bounds are those of ops_ref.py."""
import numpy as np

import ops_ref as R

ROOT, NONE = -1, -2


def ancestry(parents):
    """parents of one tree -> (rows that are in it [q], what each has in front of it and itself [q, q])"""
    q = len(parents)
    inside, family = np.zeros(q, bool), np.zeros((q, q), bool)
    for j, p in enumerate(parents):
        if p == ROOT:
            inside[j] = True
        elif 0 <= p < j:
            inside[j] = inside[p]
            family[j] = family[p]
        if inside[j]:
            family[j, j] = True
        else:
            family[j] = False
    return inside, family


def depth(parents):
    """Ancestors of each row; 0 of rows that are in no tree."""
    inside, family = ancestry(parents)
    return np.where(inside, family.sum(1) - 1, 0)


def sight(length, new, parents):
    """[new, length]: which cached tokens each new one sees; parents None: the new tokens follow one another."""
    seen = np.zeros((new, length), bool)
    if length == 0:
        return seen
    base = length - new
    if parents is None:
        return np.arange(length)[None] <= base + np.arange(new)[:, None]
    inside, family = ancestry(parents)
    seen[:, :base] = inside[:, None]
    seen[:, base:] = family
    return seen


def attention(pool_layer, tables, lens, q_lens, parents, q, scale, io, B):
    """As ops_ref.attention; parents: of each request a list, or None."""
    H, D = pool_layer.shape[3], pool_layer.shape[4]
    T, Hq = q.shape[:2]
    G, u = Hq // H, R.U[io]
    out, tol = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, ltol = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    weights, wtol = [], []
    t = 0
    for table, length, new, tree in zip(tables, lens, q_lens, parents):
        kv = R.request_rows(pool_layer, table, length, B)
        w, wt = np.zeros((H, length)), np.zeros((H, length))
        seen = sight(length, new, tree)
        live = seen.any(1)
        used = seen.any(0)
        kv = np.where(used[None, :, None, None], kv, 0.0)  # (what nobody sees may be anything)
        for h in range(H if live.any() else 0):
            k, v = kv[0, :, h], kv[1, :, h]
            rows = np.where(live[:, None, None], q[t:t + new, h * G:(h + 1) * G], 0.0)  # [new, G, D]
            z = rows @ k.T * scale
            mag = np.abs(rows) @ np.abs(k).T * abs(scale)
            z = np.where(seen[:, None], z, -np.inf)
            mag = np.where(seen[:, None], mag, 0.0)
            m = np.where(live[:, None], z.max(-1), 0.0)
            ds = (D + 4) * 2.0 ** -23 * mag.max(-1) + 2.0 ** -22 * np.where(seen[:, None], np.abs(np.where(seen[:, None], z, 0)), 0).max(-1) + 2.0 ** -20
            e = np.exp(z - m[..., None])
            total = np.where(live[:, None], e.sum(-1), 1.0)
            p = e / total[..., None]
            o = p @ v
            spread = p @ np.abs(v)
            count = seen.sum(1)[:, None]
            at = (slice(t, t + new), slice(h * G, (h + 1) * G))
            out[at] = np.where(live[:, None, None], o, 0.0)
            tol[at] = np.where(live[:, None, None], u * np.abs(o) + spread * (u + 2 * ds + (count + 64) * 2.0 ** -23)[..., None] + 1e-30, 0.0)
            lse[at] = np.where(live[:, None], m + np.log(total), -np.inf)
            ltol[at] = np.where(live[:, None], 2 * ds + 2.0 ** -22 * (1 + np.abs(m + np.log(total))), 0.0)
            w[h] = p.sum((0, 1))
            wt[h] = (p * (4 * ds + 2.0 ** -20)[..., None]).sum((0, 1))
        t += new
        weights.append(w)
        wtol.append(wt)
    return out, tol, lse, ltol, weights, wtol


def accepted(parents, tokens, chosen):
    """One request's path, and the token that follows it."""
    inside, _ = ancestry(parents)
    path = []
    u = 0 if len(parents) and inside[0] else None
    while u is not None:
        path.append(u)
        u = next((j for j in range(u + 1, len(parents)) if parents[j] == u and tokens[j] == chosen[u]), None)
    return path, int(chosen[path[-1]]) if path else -1


def rotate_axes(x, positions, pair_axes, freq_turns, magnitude, interleaved):
    """As ops_ref.rotate with positions [axes, T]: every pair by the position on its own axis."""
    rot = 2 * len(freq_turns)
    y, mag = x.copy(), np.abs(x)
    word = np.round(np.asarray(freq_turns, np.longdouble) * np.longdouble(2) ** 64).astype(object)
    for t in range(x.shape[0]):
        ang = np.array([(int(w) * int(positions[a, t])) % (1 << 64) / 2.0 ** 64 for w, a in zip(word, pair_axes)]) * 2 * np.pi
        c, s = np.cos(ang) * magnitude, np.sin(ang) * magnitude
        a_at = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
        b_at = a_at + 1 if interleaved else a_at + rot // 2
        a, b = x[t][:, a_at], x[t][:, b_at]
        y[t][:, a_at], y[t][:, b_at] = a * c - b * s, b * c + a * s
        mag[t][:, a_at] = mag[t][:, b_at] = (np.abs(a) + np.abs(b)) * abs(magnitude)
    return y, mag

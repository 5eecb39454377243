"""A step of drafted tokens written out in 64 bits on the CPU, one definition at a time (include/festina.h): what the GPU
tests compare with.  Loops over requests and nodes; no code of the library."""
import numpy as np

import kv_reference as K

MOST = 64


def tree(rng, n, spread):
    """Parents of a random tree of n nodes: each of the `spread` before it."""
    return [-1] + [i - 1 - int(rng.integers(0, min(i, spread))) for i in range(1, n)] if n else []


def paths(parent, n):
    """Each node's line from the root, itself included (a parent that is not an earlier node counts as none)."""
    out = []
    for i in range(n):
        p = int(parent[i])
        out.append((out[p] if 0 <= p < i else []) + [i])
    return out


def plan(first, length, parent):
    """(seen as Python integers, position); tokens of no request are None."""
    T = len(parent)
    seen, position = [None] * T, [None] * T
    for r in range(len(length)):
        f, n = int(first[r]), int(first[r + 1] - first[r])
        before = int(length[r]) - n
        for i, line in enumerate(paths(parent[f:f + n], n) if n <= MOST else []):
            seen[f + i], position[f + i] = sum(1 << j for j in line), before + len(line) - 1
        for i in range(n if n > MOST else 0):
            seen[f + i], position[f + i] = 0, before + i
    return seen, position


def accept(first, length, parent, token, choice):
    """(path, kept, next, length); tokens of no request are None."""
    path, kept, after, left = [None] * len(parent), [], [], []
    for r in range(len(length)):
        f, n = int(first[r]), int(first[r + 1] - first[r])
        p = list(range(n)) if n > MOST else [0] if n else []
        while 0 < n <= MOST:
            child = [c for c in range(1, n) if parent[f + c] == p[-1] and p[-1] < c and token[f + c] == choice[f + p[-1]]]
            if not child:
                break
            p.append(child[0])
        for i in range(n):
            path[f + i] = p[i] if i < len(p) else -1
        kept.append(len(p))
        after.append(int(choice[f + p[-1]]) if n else -1)
        left.append(int(length[r]) - n + len(p))
    return path, kept, after, left


def keep(k_codes, v_codes, k_scale, v_scale, table, length, first, path, kept):
    """The caches with the kept tokens moved together (requests that the definition leaves alone are left)."""
    out = [np.array(k_codes), np.swapaxes(np.array(v_codes), 2, 3).copy(), np.array(k_scale), np.array(v_scale)]
    n_blocks, _, bt, _ = out[0].shape
    for r in range(len(length)):
        n, L = int(first[r + 1] - first[r]), int(length[r])
        before, k = L - n, min(int(kept[r]), n)
        p = [int(x) for x in path[int(first[r]):int(first[r]) + max(k, 0)]]
        if n > MOST or k < 1 or before < 0 or L > table.shape[1] * bt:
            continue
        if any(not 0 <= x < n for x in p) or any(x >= y for x, y in zip(p, p[1:])):
            continue
        if any(not 0 <= table[r][c] < n_blocks for c in range(before // bt, (L - 1) // bt + 1)):
            continue
        for codes, scale in ((out[0], out[2]), (out[1], out[3])):
            was, had = codes.copy(), scale.copy()
            for c in range(before // bt, (before + k - 1) // bt + 1):
                b = int(table[r][c])
                here = [(o, o if o < before else before + p[o - before]) for o in range(c * bt, min(before + k, (c + 1) * bt))]
                came = [int(table[r][s // bt]) for o, s in here]
                for h in range(codes.shape[1]):
                    now = max(float(had[x, h]) for x in came)
                    scale[b, h] = now
                    for (o, s), x in zip(here, came):
                        codes[b, h, o % bt] = K.encode(K.decode(was[x, h, s % bt]) * (float(had[x, h]) / now))
    return out[0], np.swapaxes(out[1], 2, 3), out[2], out[3]


def trim(held, keep_, table, free_ids, n_free, block_tokens):
    """(free_ids, length, n_free)."""
    out, length = list(free_ids), np.array(held, np.int32)
    n = min(max(int(n_free), 0), len(out))
    for r in range(len(held)):
        h, k = int(held[r]), int(keep_[r])
        if not 0 <= k <= h:
            continue
        length[r] = k
        if h > table.shape[1] * block_tokens:
            continue
        for c in range(-(-k // block_tokens), -(-h // block_tokens)):
            if n < len(out):
                out[n] = table[r][c]
                n += 1
    return np.array(out, np.int32), length, n


def rotate(x, position, freq, weight=None, eps=1e-6, interleaved=False):
    """(y, bound): x [T][heads][D] in float64 as the definition has it, the angles in long doubles, and what float32
    arithmetic may be off by before the last rounding.

    With u = 2^-24: the mean's sum of D squares is off by at most D u of itself, so the factor 1 / sqrt by D u / 2 and 4 u of
    the mean's division, the sum with eps, the root and the quotient; two products per element add 2 u.  A cosine and a
    sine: the part of a turn is rounded once (u of at most pi radians), the functions are off by at most 2 units in the last
    place (4 u), a frequency's rounding to 2^-64 turns makes at most 2^31 2^-65 turns.  Each of the two products and the sum of
    a rotation rounds by u."""
    x = np.asarray(x, np.float64)
    D, half = x.shape[-1], len(freq)
    u = 2.0 ** -24
    y, rel = x.copy(), 0.0
    if weight is not None:
        y = y / np.sqrt(np.mean(y * y, -1, keepdims=True) + eps) * np.asarray(weight, np.float64)
        rel = (D / 2 + 6) * u
    size = np.abs(y)
    if half:
        turn = np.longdouble("6.28318530717958647692528676655900577")
        angle = np.asarray(position, np.longdouble)[:, None] * np.asarray(freq, np.float64).astype(np.longdouble)
        angle = angle - np.round(angle / turn) * turn
        c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
        i = np.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        p, q = y[..., a].copy(), y[..., b].copy()
        y[..., a], y[..., b] = p * c - q * s, q * c + p * s
        both = np.abs(p) + np.abs(q)
        size[..., a] = size[..., b] = both
        rel = rel + (np.pi + 4 + 3) * u + 2 * np.pi * 2.0 ** -34
    return y, size * rel


def attend(q, k_codes, v_codes, k_scale, v_scale, table, length, first, seen, scale, window=0):
    """As kv_reference.attend, for drafted tokens (seen: Python integers): (out, lse, magnitude).  A row that sees a NaN among the
    keys' codes is NaN, one that sees a NaN among the values' has NaN there."""
    T, heads, D = q.shape
    n_blocks, H, bt, _ = k_codes.shape
    G = heads // H
    out, lse = np.full((T, heads, D), np.nan), np.full((T, heads), np.nan)
    mag, vmax, logit, keys = np.zeros((T, heads, D)), np.zeros((T, heads, D)), np.zeros((T, heads)), np.zeros((T, heads))
    with np.errstate(all="ignore"):
        for r in range(len(length)):
            n, L = int(first[r + 1] - first[r]), int(length[r])
            before, cols = L - n, -(-L // bt)
            ids = np.asarray(table[r][:cols], np.int64)
            there = np.repeat((ids >= 0) & (ids < n_blocks), bt)[:L]
            ids = np.where((ids >= 0) & (ids < n_blocks), ids, 0)
            j = np.arange(L)
            see = []
            for i in range(n):
                if n > MOST:
                    s = j <= before + i
                    p = before + i
                    if window:
                        s &= j > p - window
                else:
                    nodes = [x for x in range(n) if seen[int(first[r]) + i] >> x & 1]
                    p = before + max(len(nodes) - 1, 0)
                    s = j < before
                    if window:
                        s &= j > p - window
                        nodes = nodes[-window:]
                    for x in nodes:
                        if before + x >= 0:
                            s[before + x] = True
                see.append(s & there)
            for h in range(H):
                Kx = (K.decode(k_codes[ids, h]) * k_scale[ids, h].astype(np.float64)[:, None, None]).reshape(-1, D)[:L]
                V = np.swapaxes(K.decode(v_codes[ids, h]), 1, 2) * v_scale[ids, h].astype(np.float64)[:, None, None]
                V = V.reshape(-1, D)[:L]
                sc = np.repeat(np.maximum(v_scale[ids, h].astype(np.float64), 2.0 ** -32), bt)[:L]
                for i in range(n):
                    t = int(first[r]) + i
                    for y in range(h * G, (h + 1) * G):
                        if not see[i].any():
                            out[t, y], lse[t, y] = 0.0, -np.inf
                            continue
                        ks, vs, qq = Kx[see[i]], V[see[i]], q[t, y].astype(np.float64)
                        x = scale * (ks @ qq)
                        m = x.max()
                        e = np.exp(x - m)
                        w = e / e.sum()
                        out[t, y], lse[t, y] = w @ vs, m + np.log(e.sum())
                        mag[t, y] = w @ np.abs(vs)
                        vmax[t, y] = np.abs(vs / sc[see[i]][:, None]).max(0) * sc[see[i]].max()
                        logit[t, y] = (np.abs(scale) * (np.abs(ks) @ np.abs(qq))).max()
                        keys[t, y] = see[i].sum()
    return out, lse, (mag, vmax, logit, keys)

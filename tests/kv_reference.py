"""The serving step's operators written out in 64 bits on the CPU, one definition at a time
(include/festina.h): what the GPU tests compare with.  Loops over requests, runs and heads; no code of
the library."""
import numpy as np

NAN_CODES = (0x7F, 0xFF)


def _decode_table():
    """The 256 values of e4m3: sign, 4 exponent bits (bias 7), 3 fraction bits; no infinities, NaN at 0x7f, 0xff."""
    t = np.empty(256, np.float64)
    for c in range(256):
        sign, e, f = -1.0 if c & 0x80 else 1.0, (c >> 3) & 15, c & 7
        t[c] = np.nan if (c & 0x7F) == 0x7F else sign * (f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
    return t


DECODE = _decode_table()


def decode(codes):
    return DECODE[np.asarray(codes, np.uint8)]


def encode(x):
    """Nearest e4m3 code of each value (a tie goes to the even code); beyond 448 saturates, not finite is NaN."""
    x = np.asarray(x, np.float64)
    up = DECODE[:0x7F]                                            # the non-negative values, ascending
    a = np.minimum(np.where(np.isfinite(x), np.abs(x), 0.0), 448.0)
    hi = np.searchsorted(up, a).clip(0, len(up) - 1)              # least value >= a
    lo = np.maximum(hi - 1, 0)
    below, above = a - up[lo], up[hi] - a
    c = np.where(a == up[hi], hi, np.where(below < above, lo, np.where(below > above, hi, np.where(lo % 2 == 0, lo, hi))))
    c = c + np.where(np.signbit(x), 0x80, 0)
    return np.where(np.isfinite(x), c, 0x7F).astype(np.uint8)


def same_codes(a, b):
    """Equal as values: NaN with either sign is one value, -0 and 0 are two."""
    a, b = np.asarray(a, np.uint8), np.asarray(b, np.uint8)
    return bool(np.all((a == b) | (((a & 0x7F) == 0x7F) & ((b & 0x7F) == 0x7F))))


# ------------------------------------------------------------------ blocks

def extend(held, add, table, free_ids, n_free, block_tokens, max_tokens):
    """(table, slot, first, length, served, n_free): the requests one after the other."""
    bt, table = block_tokens, np.array(table, np.int32)
    n_blocks = len(free_ids)
    n_free = min(max(int(n_free), 0), n_blocks)
    R, columns = table.shape
    slot = np.full(max_tokens, -1, np.int32)
    first = np.zeros(R + 1, np.int32)
    length = np.array(held, np.int32)
    served = np.zeros(R, np.uint8)
    blocks = tokens = used = filled = 0
    for r in range(R):
        h, a = int(held[r]), int(add[r])
        first[r] = filled
        if h < 0 or a < 0 or h + a > columns * bt:
            continue
        have, total = -(-h // bt), -(-(h + a) // bt)
        blocks, tokens = blocks + total - have, tokens + a
        if blocks > n_free or tokens > max_tokens:
            continue
        for c in range(have, total):
            table[r, c] = free_ids[n_free - 1 - used]
            used += 1
        for p in range(h, h + a):
            b = int(table[r, p // bt])
            if 0 <= b < n_blocks:
                slot[filled] = b * bt + p % bt
            filled += 1
        length[r], served[r] = h + a, 1
    first[R] = filled
    return table, slot, first, length, served, n_free - used


def release(held, done, table, free_ids, n_free, block_tokens):
    """(free_ids, length, n_free)."""
    out, length = list(free_ids), np.array(held, np.int32)
    n = min(max(int(n_free), 0), len(out))
    for r in range(len(held)):
        if not done[r]:
            continue
        if 0 <= held[r] <= table.shape[1] * block_tokens:
            for c in range(-(-int(held[r]) // block_tokens)):
                if n < len(out):
                    out[n] = table[r][c]
                    n += 1
        length[r] = 0
    return np.array(out, np.int32), length, n


# ------------------------------------------------------------------ the cache

def scale_of(amax):
    """The least power of two s with amax <= 448 s, within [2^-32, 2^32]."""
    s = 2.0 ** -32
    while s < 2.0 ** 32 and amax > 448 * s:
        s *= 2
    return s


def store(k_codes, v_codes, k_scale, v_scale, k, v, slot, block_tokens):
    """The updated (k_codes, v_codes, k_scale, v_scale); v_codes with tokens last."""
    bt = block_tokens
    out = [np.array(k_codes), np.swapaxes(np.array(v_codes), 2, 3).copy(), np.array(k_scale), np.array(v_scale)]
    n_slots, t, T = out[0].shape[0] * bt, 0, len(slot)
    while t < T:
        s, n = int(slot[t]), 1
        if not 0 <= s < n_slots:
            t += 1
            continue
        while t + n < T and slot[t + n] == s + n and (s + n) % bt:
            n += 1
        b, o = divmod(s, bt)
        for x, codes, scale in ((k, out[0], out[2]), (v, out[1], out[3])):
            for h in range(x.shape[1]):
                y = np.asarray(x[t:t + n, h], np.float64)
                now = scale_of(np.max(np.abs(np.where(np.isfinite(y), y, 0.0))))
                old = float(scale[b, h])
                if o:
                    now = max(now, old)
                    if now > old:
                        codes[b, h, :o] = encode(decode(codes[b, h, :o]) * (old / now))
                codes[b, h, o:o + n] = encode(y / now)
                scale[b, h] = now
        t += n
    return out[0], np.swapaxes(out[1], 2, 3), out[2], out[3]


# ------------------------------------------------------------------ attention

def attend(q, k_codes, v_codes, k_scale, v_scale, table, length, first, scale, window=0):
    """(out, lse, magnitude): float64 [T][heads][D], [T][heads]; magnitude holds, for the bounds on rounding,
    per row sum_j w_j |v_j| [T][heads][D], the largest |code| times the largest scale of the values seen
    [T][heads][D], max_j scale sum_d |q_d k_jd| and the number of keys.  Rows of no request are NaN."""
    T, heads, D = q.shape
    n_blocks, H, bt, _ = k_codes.shape
    G = heads // H
    out, lse = np.full((T, heads, D), np.nan), np.full((T, heads), np.nan)
    mag, vmax, logit, keys = np.zeros((T, heads, D)), np.zeros((T, heads, D)), np.zeros((T, heads)), np.zeros((T, heads))
    with np.errstate(all="ignore"):
        for r in range(len(length)):
            n = int(first[r + 1] - first[r])
            L = int(length[r])
            cols = -(-L // bt)
            ids = np.asarray(table[r][:cols], np.int64)
            there = np.repeat((ids >= 0) & (ids < n_blocks), bt)[:L]
            ids = np.where((ids >= 0) & (ids < n_blocks), ids, 0)
            for h in range(H):
                K = (decode(k_codes[ids, h]) * k_scale[ids, h].astype(np.float64)[:, None, None]).reshape(-1, D)[:L]
                V = np.swapaxes(decode(v_codes[ids, h]), 1, 2) * v_scale[ids, h].astype(np.float64)[:, None, None]
                V = V.reshape(-1, D)[:L]
                sc = np.repeat(np.maximum(v_scale[ids, h].astype(np.float64), 2.0 ** -32), bt)[:L]
                for i in range(n):
                    p = L - n + i
                    j = np.arange(L)
                    see = (j <= p) & there
                    if window:
                        see &= j > p - window
                    t = int(first[r]) + i
                    for y in range(h * G, (h + 1) * G):
                        if not see.any():
                            out[t, y], lse[t, y] = 0.0, -np.inf
                            continue
                        ks, vs, qq = K[see], V[see], q[t, y].astype(np.float64)
                        x = scale * (ks @ qq)
                        m = x.max()
                        e = np.exp(x - m)
                        w = e / e.sum()
                        out[t, y], lse[t, y] = w @ vs, m + np.log(e.sum())
                        mag[t, y] = w @ np.abs(vs)
                        vmax[t, y] = np.abs(vs / sc[see][:, None]).max(0) * sc[see].max()
                        logit[t, y] = (np.abs(scale) * (np.abs(ks) @ np.abs(qq))).max()
                        keys[t, y] = see.sum()
    return out, lse, (mag, vmax, logit, keys)


def attend_bounds(out, lse, magnitude, dim, half_ulp):
    """How far a kernel may be that forms logits in float32 from exact products, takes the weights (relative to
    the largest of a row) in half precision and sums in float32; `half_ulp` is the output type's unit roundoff.

    A logit is off by at most dx = (D + 4) 2^-24 X (its sum of D products of total magnitude X, the scaling and the
    shift), so a weight by a factor exp(2 dx); exponential and division add under 2^-20.  A weight's rounding is
    2^-11 of it, or 2^-25 of the row's largest where it is subnormal (weights multiply codes and carry their
    block's scale, the largest included).  The float32 sum over n keys adds n 2^-24."""
    mag, vmax, logit, keys = magnitude
    dx = (dim + 4) * 2.0 ** -24 * logit
    rel = 2.0 ** -11 + 2 * dx + 2.0 ** -20 + keys * 2.0 ** -24
    tol_out = half_ulp * np.abs(out) + 1.01 * mag * rel[..., None] + (keys * 2.0 ** -25)[..., None] * vmax + 1e-30
    tol_lse = dx + 2.0 ** -20 + keys * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse)
    return tol_out, tol_lse

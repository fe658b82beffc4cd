"""Plain 64-bit implementations of the cache operators, and their inputs (CPU, numpy)."""

import numpy as np

E4M3_MAX = 448.0


def code_values():
    """[256] what each e4m3 code stands for (4-bit exponent of bias 7, 3-bit mantissa, no infinities)."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = np.nan if c & 127 == 127 else m * 2.0**-9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = -x if c & 128 else x
    return v


VALUES = code_values()


def nearest_code(x):
    """Codes of finite x (|x| <= 448): nearest value, ties to the even code."""
    pos = VALUES[:127]
    a = np.abs(x)
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (pick + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_for(amax):
    """Least power of two s >= 2^-126 with amax <= 448 s; 0 for 0."""
    a = np.asarray(amax, np.float64)
    with np.errstate(divide="ignore"):
        s = np.exp2(np.ceil(np.log2(a / E4M3_MAX)))
    return np.where(a > 0, np.maximum(s, 2.0**-126), 0.0)


def rotate(x, pos, cos, sin, interleaved):
    """x [tokens, heads, dim], cos / sin [positions, rot / 2]; 64 bits."""
    y = np.array(x, np.float64)
    half = cos.shape[1]
    i = np.arange(half)
    lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    c, s = cos[pos].astype(np.float64)[:, None], sin[pos].astype(np.float64)[:, None]
    a, b = y[..., lo].copy(), y[..., hi].copy()
    y[..., lo] = a * c - b * s
    y[..., hi] = b * c + a * s
    return y


def attend(q, k_codes, v_codes, k_scale, v_scale, table, length, q_start, scale, window):
    """(out [tokens, q_heads, dim], sum p |v|, largest sum |q k| scale per row) in 64 bits.
    Caches [pages, heads, P, dim] of codes."""
    T, Hq, D = q.shape
    _, H, P, _ = k_codes.shape
    G = Hq // H
    out, mag, dots = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq, 1))
    for b in range(len(length)):
        L, n0, n1 = int(length[b]), int(q_start[b]), int(q_start[b + 1])
        n = n1 - n0
        if n == 0 or L <= 0:
            continue
        at = table[b, : -(-L // P)]
        pos = np.arange(L - n, L)
        j = np.arange(L)
        seen = j[None] <= pos[:, None]
        if window:
            seen &= j[None] > pos[:, None] - window
        for h in range(H):
            k = (VALUES[k_codes[at, h]] * k_scale[at, h].astype(np.float64)[:, None, None]).reshape(-1, D)[:L]
            v = (VALUES[v_codes[at, h]] * v_scale[at, h].astype(np.float64)[:, None, None]).reshape(-1, D)[:L]
            for g in range(h * G, (h + 1) * G):
                x = q[n0:n1, g].astype(np.float64) @ k.T * scale
                x = np.where(seen, x, -np.inf)
                top = x.max(1, keepdims=True, initial=-np.inf)
                p = np.exp(x - np.where(np.isfinite(top), top, 0.0))
                total = p.sum(1, keepdims=True)
                p /= np.where(total > 0, total, 1.0)
                out[n0:n1, g] = p @ v
                mag[n0:n1, g] = p @ np.abs(v)
                dots[n0:n1, g, 0] = (np.abs(q[n0:n1, g].astype(np.float64)) @ np.abs(k.T) * np.where(seen, 1.0, 0.0)
                                     ).max(1) * abs(scale)
    return out, mag, dots


def make(rng, lens, heads, dim, page, spare=2, spread=0.5):
    """Random caches and tables for sequences of (length, new) tokens: codes [pages, heads, page,
    dim], power-of-two scales, a shuffled page table."""
    need = [max(0, -(-l // page)) for l, _ in lens]
    pages = sum(need) + spare
    perm = rng.permutation(pages).astype(np.int32)
    width = max(1, max(need))
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for b, c in enumerate(need):
        table[b, :c] = perm[at : at + c]
        at += c
    out = {"table": table, "length": np.array([l for l, _ in lens], np.int32),
           "q_start": np.concatenate([[0], np.cumsum([n for _, n in lens])]).astype(np.int32), "pages": pages}
    for n in ("k", "v"):
        x = rng.standard_normal((pages, heads, page, dim)) * np.exp(spread * rng.standard_normal((pages, heads, 1, 1)))
        s = scale_for(np.abs(x).max((2, 3)))
        out[n] = nearest_code(x / s[:, :, None, None])
        out[n + "_scale"] = s.astype(np.float32)
    return out

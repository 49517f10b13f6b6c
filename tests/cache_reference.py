"""Plain 64-bit forms of the operators around the 8-bit paged cache, written from their definitions: rotary positions, the
append of keys and values, attention over the cache.  Test infrastructure; shares no code with the library."""
import math

import numpy as np

BLOCK, DH = 64, 64


def e4m3_table():
    """The 256 values of the format, from its bit fields (sign 1, exponent 4 with bias 7, mantissa 3; 0x7f and 0xff: no number)."""
    out = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, c >> 3 & 15, c & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[c] = math.nan if e == 15 and m == 7 else -v if s else v
    return out


VALUES = e4m3_table()
_POS = VALUES[:127]                                   # 0 .. 448, ascending


def to_code(x):
    """Nearest E4M3 code, ties to the even code, saturating; NaN: 0x7f."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0, x)), 448.0)
    hi = np.searchsorted(_POS, a)                     # _POS[hi - 1] < a <= _POS[hi]
    lo = np.maximum(hi - 1, 0)
    up, down = _POS[hi] - a, a - _POS[lo]
    c = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return np.where(np.isnan(x), 0x7F, c | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def fresh_scale(x):
    """Least power of two >= 2^-126 that brings the finite values of x within 448."""
    a = np.abs(np.asarray(x, np.float64))
    top = a[np.isfinite(a)].max(initial=0.0)
    e = -126
    while top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append(codes, scales, table, k, v, row_start, n_new, pos_start):
    """In place; codes uint8 [blocks, heads, 2, 4096], scales [blocks, heads, 2]; k, v float [rows, heads, 64]."""
    for b in range(len(n_new)):
        p, end, row = int(pos_start[b]), int(pos_start[b] + n_new[b]), int(row_start[b])
        while p < end:
            blk, lo = p // BLOCK, p % BLOCK
            hi = min(BLOCK, lo + end - p)
            at = int(table[b, blk])
            for h in range(codes.shape[1]):
                for w, x in ((0, k), (1, v)):
                    new = np.asarray(x[row:row + hi - lo, h], np.float64)
                    s = fresh_scale(new)
                    body = codes[at, h, w].reshape(BLOCK, DH) if w == 0 else codes[at, h, w].reshape(DH, BLOCK).T      # [token, dim], views
                    if lo > 0:
                        s = max(s, float(scales[at, h, w]))
                        if s != scales[at, h, w]:
                            body[:lo] = to_code(VALUES[body[:lo]] * (float(scales[at, h, w]) / s))
                    body[lo:hi] = to_code(new / s)
                    scales[at, h, w] = s
            row += hi - lo
            p += hi - lo


def rotate(x, positions, turns, amplitude, interleaved, inverse):
    """float64 [tokens, heads, dims]; the fraction of a turn from exact integer arithmetic on the double `turns`."""
    from fractions import Fraction
    x = np.array(x, np.float64)
    r = 2 * len(turns)
    frac = np.array([[float(Fraction(float(t)) * int(p) % 1) for t in turns] for p in positions]).reshape(len(positions), r // 2)
    ang = 2 * math.pi * frac * (-1 if inverse else 1)
    c, s = (np.cos(ang) * amplitude)[:, None], (np.sin(ang) * amplitude)[:, None]
    ia, ib = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., ia].copy(), x[..., ib].copy()
    x[..., ia], x[..., ib] = a * c - b * s, a * s + b * c
    return x


def attend(q, codes, scales, table, n_rows, lens, scale, spans=None, bias=None, cap=0.0):
    """q float [batch, rows, heads * 64] -> (out, softmax over |v|, bound on what rounding may do but for the output's and the weights' own), float64.

    The bound, from the arithmetic the documentation states.  A score is a sum of 64 products in fp32 (each addition off by at most 2^-23
    of what is summed: 2^-17 in all) of f16 parts of q (bf16: one, exact; fp32: two, off by 2^-22), off by 2^-24 of the row's largest where f16 runs out of exponents; its scaling, cap
    (tanh within 2^-21) and bias add 2^-21 of each.  A weight is then off by twice the score's error (its own and the sum's) and by the
    rounding of weights (relative: the caller's, times the second result; absolute: weights are 2^15 times their share of the block's largest in f16, whose
spacing is never below 2^-24, so half of it is 2^-40 of the largest); the weighted sum of values by 2^-16 more (64 products per block, then one
addition per block)."""
    batch, rows, width = q.shape
    heads, kv = width // DH, codes.shape[1]
    out, slack, mean = np.zeros((batch, rows, heads, DH)), np.zeros((batch, rows, heads, DH)), np.zeros((batch, rows, heads, DH))
    for b in range(batch):
        n = int(lens[b])
        if n == 0:
            continue
        at = table[b, :-(-n // BLOCK)]
        val = VALUES[codes[at]] * np.asarray(scales, np.float64)[at][..., None]
        K = val[:, :, 0].reshape(-1, kv, BLOCK, DH).transpose(1, 0, 2, 3).reshape(kv, -1, DH)
        V = val[:, :, 1].reshape(-1, kv, DH, BLOCK).transpose(1, 0, 3, 2).reshape(kv, -1, DH)
        for r in range(int(n_rows[b])):
            lo, hi = (0, n) if spans is None else (max(int(spans[b, r, 0]), 0), min(int(spans[b, r, 1]), n))
            if lo >= hi:
                continue
            for h in range(heads):
                qq, k, v = np.asarray(q[b, r, h * DH:(h + 1) * DH], np.float64), K[h * kv // heads, lo:hi], V[h * kv // heads, lo:hi]
                s = scale * (k @ qq)
                err = scale * ((2.0 ** -17 + 2.0 ** -22) * (np.abs(k) @ np.abs(qq)) + 2.0 ** -24 * np.abs(qq).max() * np.abs(k).sum(-1)) + 2.0 ** -21 * np.abs(s)
                if cap > 0:
                    s = cap * np.tanh(s / cap)
                    err = err + 2.0 ** -21 * cap
                if bias is not None:
                    add = np.asarray(bias, np.float64)[h, np.minimum(hi - 1 - np.arange(lo, hi), bias.shape[1] - 1)]
                    s = s + add
                    err = err + 2.0 ** -21 * (np.abs(add) + np.abs(s))
                w = np.exp(s - s.max())
                w /= w.sum()
                out[b, r, h] = w @ v
                mean[b, r, h] = w @ np.abs(v)
                slack[b, r, h] = mean[b, r, h] * (2 * err.max() + 2.0 ** -16) + 2.0 ** -40 * np.abs(v).sum(0)
    flat = lambda a: a.reshape(batch, rows, width)  # noqa: E731
    return flat(out), flat(mean), flat(slack)

"""Plain 64-bit forms of the operators over contexts kept in 8 bits, in numpy, written from their definitions; no code of the library."""
import math

import numpy as np

MOST = {"int8": 127.0, "e4m3": 448.0}
# every finite number of 8 bits with 4 of exponent and 3 of mantissa, in rising order
E4M3 = np.array(sorted({s * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) for s in (1, -1) for e in range(16) for m in range(8) if (e, m) != (15, 7)}))


def turned(x, w, eps, pos, freq, interleaved, amplitude):
    """Norm (w None: none) and rotation (freq None: none) of x [n, heads, D] float64."""
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    if freq is None:
        return x
    y, half = x.copy(), len(freq)
    ang = np.asarray(pos, dtype=np.float64)[:, None, None] * freq
    c, s = amplitude * np.cos(ang), amplitude * np.sin(ang)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def exponent(top, most):
    """The smallest e >= -100 with top <= most 2^e; -128 for what is no number."""
    if not math.isfinite(top):
        return -128
    e = -100
    while top > most * 2.0 ** e:
        e += 1
    return e


def quantized(x, kind):
    """Values (as numbers) and exponents of x [n, heads, D] float64."""
    with np.errstate(invalid="ignore"):
        top = np.where(np.isfinite(x).all(-1), np.abs(x).max(-1), np.inf)
    e = np.array([[exponent(t, MOST[kind]) for t in row] for row in top], dtype=np.int64).reshape(top.shape)
    y = np.where((e == -128)[..., None], 0.0, x) * 2.0 ** -np.where(e == -128, 0, e)[..., None].astype(np.float64)
    return (np.rint(y) if kind == "int8" else nearest_e4m3(y)), e


def nearest_e4m3(y):
    """To the nearest number of the type, of two as near the one with the even mantissa."""
    hi = np.clip(np.searchsorted(E4M3, y), 0, len(E4M3) - 1)
    lo = np.maximum(hi - 1, 0)
    a, b = y - E4M3[lo], E4M3[hi] - y
    step = lambda v: np.exp2(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6))) - 3)
    even = (np.round(E4M3[lo] / step(E4M3[lo])) % 2) == 0
    return np.where((a < b) | ((a == b) & even), E4M3[lo], E4M3[hi])


def values(v, e):
    """What values [.., D] and exponents [..] stand for."""
    return np.where((e == -128)[..., None], np.nan, v * 2.0 ** np.where(e == -128, 0, e)[..., None].astype(np.float64))


def attention(q, k, v, lens, scale, v_scale=None):
    """q [rows, H, D], k, v [T, H_kv, D], lens [rows]: (out, lse, sum of weights times |v|, largest sum of |q k| scale, what weights of 16 bits may lose); v_scale [T, H_kv]: what
    a value's one stands for."""
    rows, H, D = q.shape
    G = H // k.shape[1] if k.shape[0] else H
    out, mass = np.zeros((rows, H, D)), np.zeros((rows, H, D))
    lse, most, lost = np.full((H, rows), -np.inf), np.zeros((H, rows)), np.zeros((H, rows))
    for r in range(rows):
        for h in range(H):
            n = lens[r]
            if n <= 0:
                continue
            kk, vv = k[:n, h // G], v[:n, h // G]
            s = kk @ q[r, h] * scale
            m = s.max()
            p = np.exp(s - m)
            z = p.sum()
            out[r, h], mass[r, h] = p @ vv / z, p @ np.abs(vv) / z
            lse[h, r], most[h, r] = m + math.log(z), (np.abs(kk) @ np.abs(q[r, h])).max() * scale
            if v_scale is not None:
                lost[h, r] = 2.0 ** -39 * n * 448 * np.nanmax(p / z * v_scale[:n, h // G])
    return out, lse, mass, most, lost


def attention_tolerance(want, lse, mass, most, lost, D):
    """(of the output, of lse).  A score is a sum of D exact products in fp32, off by at most D 2^-24 of the sum of their sizes, and rounded a few times behind it: 'a'.
    exp2 and log2 of the hardware: 2^-21 each with the rounding of their arguments' products.  A weight is rounded to fp16 (2^-11); weights are summed in fp32 by 32 and by parts:
    2^-18 for up to 2^6 roundings of the sum in turn.  The output is rounded to bf16 (2^-8).
    Where scores are off by a, a weight over the sum of all is off by a factor between e^-2a and e^2a.  And fp16 has no steps below 2^-24: with the largest weight times its value's scale at
    2^14, a weight is off by up to 2^-25 all the same, 2^-39 of that largest, for each of n tokens and values of up to 448 ('lost')."""
    a = (D + 8) * 2.0 ** -24 * most
    rel = 2.0 ** -11 + np.maximum(4 * a, np.expm1(2 * a)).T[..., None] + 2.0 ** -18
    with np.errstate(invalid="ignore"):
        lse_tol = np.where(np.isfinite(lse), a + 2.0 ** -18 + 2.0 ** -21 * np.abs(np.where(np.isfinite(lse), lse, 0)), 0.0)
    return rel * mass + 2.0 ** -8 * np.abs(want) + 2 * lost.T[..., None] + 1e-37, lse_tol

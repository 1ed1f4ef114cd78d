"""Plain 64-bit forms of the operators over continuations, in numpy, written from their definitions; no code of the library."""

import numpy as np


def block_tables(bs, seq_len, new_len, base, free, n_free, table, n_rows):
    """(row_cu, rows as (seq, pos, len, slot), seq_len, n_free, free, table) after the step, by hand."""
    table, free, seq_len = [list(r) for r in table], list(free), list(seq_len)
    width = len(table[0])
    blocks = lambda t: -(-t // bs)
    ok = [0 <= n <= width * bs and a <= n_rows and n + max(a, 0) <= width * bs for n, a in zip(seq_len, new_len)]
    back = [b for i, a in enumerate(new_len) if ok[i] and a < 0 for b in table[i][:blocks(seq_len[i])]]
    if n_free < 0 or n_free + len(back) > len(free):
        return [0] * (len(seq_len) + 1), [], seq_len, n_free, free, table
    stack = free[:n_free] + back
    add = [a if o and a > 0 else 0 for a, o in zip(new_len, ok)]
    need = sum(blocks(n + a) - blocks(n) for n, a in zip(seq_len, add))
    if sum(add) > n_rows or need > len(stack):
        add = [0] * len(add)
    rows, cu = [], [0]
    for i, a in enumerate(add):
        if ok[i] and new_len[i] < 0:
            seq_len[i] = 0
        for _ in range(a):
            t = seq_len[i]
            if t % bs == 0:
                table[i][t // bs] = stack.pop()
            rows.append((i, base[i] + t, t + 1, table[i][t // bs] * bs + t % bs))
            seq_len[i] += 1
        cu.append(len(rows))
    for j in range(n_free, len(stack)):
        free[j] = stack[j]
    return cu, rows, seq_len, len(stack), free, table


def norm_rope(x, w, eps, pos, theta):
    """x [n, heads, D] float64."""
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    half = x.shape[-1] // 2
    ang = pos[:, None, None] * theta ** (-np.arange(half) / half)
    c, s = np.cos(ang), np.sin(ang)
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def pow2_scale(amax):
    """The smallest power of two s >= 2^-100 with amax <= 127 s; 1 for 0."""
    if amax == 0:
        return 1.0
    e = -100
    while amax > 127 * 2.0 ** e and e < 122:
        e += 1
    return 2.0 ** e


def bounds(k, bs):
    """k [T, Hkv, D] -> (int [nb, Hkv, 2, D], scale [nb, Hkv])."""
    nb = -(-k.shape[0] // bs)
    out, scale = np.zeros((nb, k.shape[1], 2, k.shape[2]), dtype=np.int64), np.zeros((nb, k.shape[1]))
    for x in range(nb):
        part = k[x * bs:(x + 1) * bs]
        for g in range(k.shape[1]):
            p = part[:, g]
            hi, lo = np.fmax.reduce(p, 0), np.fmin.reduce(p, 0)
            hi, lo = np.nan_to_num(hi, nan=0.0, posinf=np.inf, neginf=-np.inf), np.nan_to_num(lo, nan=0.0, posinf=np.inf, neginf=-np.inf)
            amax = min(np.maximum(np.abs(hi), np.abs(lo)).max(), 3.3895313892515355e38)
            s = scale[x, g] = pow2_scale(amax)
            out[x, g, 0], out[x, g, 1] = np.clip(np.ceil(hi / s), -127, 127), np.clip(np.floor(lo / s), -127, 127)
    return out, scale


def select(q, bounds_, scale, n_select, n_first, n_last):
    """q [H, D] of one row, the bounds of its context -> int [Hkv, n_select]."""
    nb, Hkv = scale.shape
    G = q.shape[0] // Hkv
    out = np.full((Hkv, n_select), -1)
    for g in range(Hkv):
        best = np.full(nb, -np.inf)
        for h in range(g * G, (g + 1) * G):
            s = pow2_scale(np.abs(q[h]).max())
            qi = np.rint(q[h] / s)
            best = np.maximum(best, (np.maximum(qi, 0) * bounds_[:, g, 0] + np.minimum(qi, 0) * bounds_[:, g, 1]).sum(-1) * s)
        best = best * scale[:, g]
        best[:n_first] = np.inf
        best[max(0, nb - n_last):] = np.inf
        order = sorted(range(nb), key=lambda x: (-best[x], x))[:n_select]
        out[g, :len(order)] = sorted(order)
    return out


def attend(q, k, v, scale):
    """One row and KV head: q [G, D], k and v [n, D] -> (out, lse, sum of the weights times |v|, largest |logit|)."""
    G, D = q.shape
    if len(k) == 0:
        return np.zeros((G, D)), np.full(G, -np.inf), np.zeros((G, D)), 0.0
    s = q @ k.T * scale
    m = s.max(-1, keepdims=True)
    p = np.exp(s - m)
    z = p.sum(-1, keepdims=True)
    return p @ v / z, (m + np.log(z))[:, 0], p @ np.abs(v) / z, np.abs(s).max()


def to_bf16(x):
    """Rounded to the nearest bf16, ties to even (by way of float32)."""
    f = np.asarray(x, dtype=np.float64).astype(np.float32)
    bits = f.view(np.uint32).astype(np.uint64)
    return ((bits + 0x7fff + ((bits >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32).astype(np.float64)


def rounded_within(got, want, delta):
    """got is the bf16 rounding of a number within delta of want (rounding keeps order)."""
    return (got >= to_bf16(want - delta)) & (got <= to_bf16(want + delta))


# Before its one rounding an output differs by the rounding of the probabilities to bf16, 8 significant bits: half a unit of the last is 2^-8 of
# the value at the most, so 2^-8 of sum w |v|; sums and exponentials in fp32 add some 1e-5 of it.
def attention_delta(abs_v):
    return 2.0 ** -8 * abs_v + 2e-5 * abs_v + 1e-30


def lse_tolerance(largest):
    """fp32: D products and sums of up to ~6 times the result's size, 2^-24 each, the logarithm of a sum of probabilities."""
    return 2e-6 * (10 + largest)



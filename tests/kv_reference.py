"""The paged K/V cache's operators from their definitions, in float64 numpy: one sequence, one head, one row at a time."""
import numpy as np


def round_e4m3(y):
    """To the nearest E4M3 number, ties to even; |y| <= 448."""
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -20))), -6) - 3)
    return np.round(y / step) * step


def quantised(x):
    """What rows (last axis) stand for once they are held as codes, and their exponents e (128: not finite)."""
    x = np.asarray(x, np.float64)
    values, exps = np.empty_like(x), np.empty(x.shape[:-1], np.int64)
    for i in np.ndindex(exps.shape):
        top = np.abs(x[i]).max()
        if not np.isfinite(top):
            values[i], exps[i] = np.nan, 128
            continue
        e = -118
        while top > 448.0 * 2.0 ** e:
            e += 1
        values[i], exps[i] = round_e4m3(x[i] * 2.0 ** -e) * 2.0 ** e, e
    return values, exps


def seen(length, rows, causal_block, i):
    if causal_block == 0:
        return length
    return max(0, min(length, length - rows + (i // causal_block + 1) * causal_block))


def attend(q, k, v, causal_block, scale):
    """q [rows, q_heads, d] over k, v [length, kv_heads, d] -> output and sum_j p_j |v_j|, both [rows, q_heads, d].  Tokens that
    a row does not see are left out, not multiplied by zero."""
    rows, q_heads, d = q.shape
    length, kv_heads = k.shape[:2]
    out, spread = np.zeros((rows, q_heads, d)), np.zeros((rows, q_heads, d))
    with np.errstate(all="ignore"):
        for h in range(q_heads):
            kh, vh = k[:, h * kv_heads // q_heads], v[:, h * kv_heads // q_heads]
            for i in range(rows):
                n = seen(length, rows, causal_block, i)
                if n == 0:
                    continue
                s = scale * (kh[:n] @ q[i, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                out[i, h] = (p[:, None] * vh[:n]).sum(0) if not np.isfinite(vh[:n]).all() else p @ vh[:n]
                spread[i, h] = p @ np.abs(vh[:n])
    return out, spread

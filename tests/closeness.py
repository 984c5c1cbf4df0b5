"""How near attention over a context in 4 bits has to come to the oracle, row by row (a query and a head each).

What is allowed follows from the roundings themselves and shrinks with the result.  A rounding with half step h is uniform in
[-h, h], so its root mean square is h / sqrt(3), and a sum of independent ones has the root of the sum of their squares.  The
norm of a row's error may be four times that: a single rounding is never above sqrt(3) times its root mean square, several
kinds at their worst in one row add up to less than four, and a norm over many strays by far less.  With a row's weights p_j
(of sum one) and token j's V = low_j + code_j * scale_j, mid_j = low_j + 8 scale_j:
  weights  bf16: p_j scale_j is rounded to 8 bits (half step 2^-8) and meets code_j - 8; f32: 24 bits (2^-24)
  minima   the weights that meet mid_j, bf16: 16 bits, of which the first eight are cut off and the rest is rounded (2^-15);
           f32: 24 bits
  scores   the score of token j is off by fp32 roundings, and an output by p_j (V_j - out) times that; some 24 of 2^-24 in a
           score, each of a partial sum of at most |q| * (16 scale of K + sqrt(D) |low of K|)
  sums     one fp32 rounding (2^-24) a token of what is being summed, whose root mean square is at most that of the summands
           in a row, and one of the exponential's result and of the weight's sum
  output   the last rounding, half step 2^-8 or 2^-24
"""
import math

import numpy as np

from oracle import q4_hold

FACTOR = 4.0


def allowed(q, held_k, held_v, lens, news, scale, bf16):
    """(reference [rows][Hq][D], bound on the norm of a row's error [rows][Hq]).  held_*: per request the result of q4_hold."""
    q = np.asarray(q, dtype=np.float64)
    n_rows, hq, d = q.shape
    ref, bound = np.zeros((n_rows, hq, d)), np.zeros((n_rows, hq))
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    half_mid = 2.0 ** -15 if bf16 else 2.0 ** -24
    row = 0
    for (k, _, k_scale, k_low), (v, code, v_scale, v_low), n, new in zip(held_k, held_v, lens, news):
        for h in range(hq if n else 0):
            kv = h // (hq // k.shape[1])
            kk, vv = k[:n, kv], v[:n, kv]
            # per token: square norms over the columns of what a rounded weight meets
            from_mid = (((code[:n, kv].reshape(n, -1, 64) - 8.0) * v_scale[:n, kv, :, None]) ** 2).sum((1, 2))
            mid = (64 * (v_low[:n, kv] + 8 * v_scale[:n, kv]) ** 2).sum(1)
            big = (16 * k_scale[:n, kv] + math.sqrt(d) * np.abs(k_low[:n, kv])).max(1)
            v_sq = (vv * vv).sum(1)
            for i in range(new):
                seen = n - new + i + 1
                if seen <= 0:
                    continue
                x = q[row + i, h]
                s = scale * (kk[:seen] @ x)
                p = np.exp(s - s.max())
                p /= p.sum()
                out = p @ vv[:seen]
                ref[row + i, h] = out
                p2, out_sq = p * p, out @ out
                e_score = 2.0 ** -24 * math.sqrt(24.0) * scale * np.linalg.norm(x) * big[:seen]
                apart = np.maximum(v_sq[:seen] - 2 * vv[:seen] @ out + out_sq, 0)
                summed = p2 @ v_sq[:seen]
                square = (half ** 2 * (p2 @ from_mid[:seen] + out_sq) + half_mid ** 2 * (p2 @ mid[:seen])
                          + 3 * (p2 * e_score ** 2) @ apart + 2.0 ** -48 * (seen + 2) * (summed + out_sq))
                bound[row + i, h] = FACTOR * math.sqrt(square / 3)
        row += new
    return ref, bound


def worst(out, ref, bound):
    """Greatest error norm of a row as a share of what is allowed (rows that see nothing have to be zeros)."""
    err = np.linalg.norm(np.asarray(out, dtype=np.float64) - ref, axis=-1)
    return float(np.where(bound > 0, err / np.where(bound > 0, bound, 1.0), np.where(err > 0, np.inf, 0.0)).max(initial=0.0))


def hold(rows, bf16):
    return [q4_hold(np.asarray(x, dtype=np.float64), bf16) for x in rows]

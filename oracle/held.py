"""Fresh rows on their way into a context, and contexts held in 4 bits, in float64 (oracle side).

The paper leaves positional embedding out (Fig. 7 caption) and names compression of the KV cache as
orthogonal to its method; the definitions are those of the public header: norms per head, rotation by
theta^(-2i/D) times the position on the pair's axis, 64 neighbouring values with a common scale and
minimum, codes 0..15.
"""
import numpy as np

GROUP = 64


def round_bf16(x):
    """Nearest bfloat16, ties to even, of finite float64 values (through float32, as the format is defined)."""
    bits = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return (((bits + 0x7FFF + (bits >> 16 & 1)) >> 16 << 16) & 0xFFFFFFFF).astype(np.uint32).view(np.float32).astype(np.float64)


def round_f32(x):
    return np.asarray(x, dtype=np.float64).astype(np.float32).astype(np.float64)


def position_rows(x, pos, theta, interleaved=False, pair_axis=None, weight=None, eps=None):
    """x [n][heads][D], pos [axes][n]; norms if eps is not None."""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    if eps is not None:
        x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
        if weight is not None:
            x = x * np.asarray(weight, dtype=np.float64)
    pos = np.asarray(pos, dtype=np.float64).reshape(-1, x.shape[0])
    out = np.empty_like(x)
    for i in range(d // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + d // 2)
        angle = pos[0 if pair_axis is None else pair_axis[i]] * float(theta) ** (-2.0 * i / d)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., a] * s + x[..., b] * c
    return out


def q4_hold(x, bf16):
    """What a cache in 4 bits holds for rows x [n][heads][D]: (values before their last rounding, codes, scales, lows)."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    with np.errstate(all="ignore"):
        low, high = g.min(axis=-1), g.max(axis=-1)
        spread = round_f32(high - low)
        bad = ~np.isfinite(spread)
        scale = round_f32(np.where(bad, 0.0, spread) / 15.0)
        if bf16:
            scale = round_bf16(scale)
        scale = np.where(scale < 2.0 ** -100, 0.0, scale)
        offset = round_f32(np.where(bad[..., None], 0.0, g - np.where(bad, 0.0, low)[..., None]))
        step = np.where(scale > 0, scale, 1.0)[..., None]
        code = np.where(scale[..., None] > 0, np.minimum(np.floor(offset / step + 0.5), 15.0), 0.0)
    scale, low = np.where(bad, np.nan, scale), np.where(bad, np.nan, low)
    value = low[..., None] + code * scale[..., None]
    return value.reshape(x.shape), code.reshape(x.shape).astype(int), scale, low


def q4_attend(q, values_k, values_v, lens, news, scale):
    """q [sum(news)][Hq][D]; values_k, values_v: per request [len][Hkv][D] as held.  Query i of a request sits at
    len - new + i.  Returns O, LSE (zeros and -inf for queries that see nothing)."""
    q = np.asarray(q, dtype=np.float64)
    nq, hq, d = q.shape
    out, lse = np.zeros((nq, hq, d)), np.full((nq, hq), -np.inf)
    row = 0
    for k, v, n, new in zip(values_k, values_v, lens, news):
        per = hq // k.shape[1] if n else 1
        for i in range(new):
            seen = n - new + i + 1
            for h in range(hq if seen > 0 else 0):
                s = scale * (k[:seen, h // per] @ q[row + i, h])
                m = s.max()
                w = np.exp(s - m)
                out[row + i, h] = w @ v[:seen, h // per] / w.sum()
                lse[row + i, h] = m + np.log(w.sum())
        row += new
    return out, lse

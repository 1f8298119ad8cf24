"""Plain forms in 64 bits of the rotary, cache and attention operators, written from their definitions, for the tests."""
import numpy as np

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}      # half a step of a rounding, relative


def turned(x, positions, theta, interleaved=False, amplitude=1.0, inverse=False):
    """x float64 [rows, heads, head_dim]"""
    y = x.copy()
    half = len(theta)
    first, second = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if interleaved else (np.arange(half), np.arange(half, 2 * half))
    angle = (-1.0 if inverse else 1.0) * positions.astype(np.float64)[:, None, None] * theta
    cos, sin = amplitude * np.cos(angle), amplitude * np.sin(angle)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
    return y


def _e4m3():
    v = []
    for code in range(127):      # 127 is the NaN
        e, m = code >> 3, code & 7
        v.append(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(v)


E4M3 = _e4m3()


def kept(x, cache):
    """what a cache holds for float64 values [..., head_dim]"""
    bad = ~np.isfinite(x).all(axis=-1, keepdims=True)
    x = np.where(bad, 0.0, x)
    if cache == "bf16":
        with np.errstate(divide="ignore"):
            e = np.where(x == 0, -126, np.maximum(np.floor(np.log2(np.abs(x))), -126))
        step = np.exp2(e - 7)
        v = np.rint(x / step) * step
    else:
        top = np.abs(x).max(axis=-1, keepdims=True)
        e = np.full(top.shape, -126.0)
        while True:      # the least power of two, by counting up
            more = top > 448 * np.exp2(e)
            if not more.any():
                break
            e = e + more
        y = np.abs(x) / np.exp2(e)
        at = np.clip(np.searchsorted(E4M3, y), 1, 126)
        low, high = E4M3[at - 1], E4M3[at]
        up = (y - low > high - y) | ((y - low == high - y) & (at % 2 == 0))       # ties to the even code
        v = np.copysign(np.where(up, high, low) * np.exp2(e), x)
    bad = bad | (np.abs(v) >= 2.0 ** 128).any(axis=-1, keepdims=True)      # rounded to what is no float32
    return np.where(bad, np.nan, v)


def attended(q, keys, values, seen, scale):
    """One sequence: q [n, heads, hd], keys and values [T, kv heads, hd], seen[i]: a boolean [n, T].  Returns the result and how far a result
    that was computed as the library says may be off: probabilities rounded to bfloat16, scores and sums in float32, one rounding at the end."""
    n, heads, hd = q.shape
    group = heads // keys.shape[1]
    out, bound = np.zeros((n, heads, hd)), np.zeros((n, heads, hd))
    for h in range(heads):
        k, v = keys[:, h // group], values[:, h // group]
        s = scale * (q[:, h] @ k.T)
        size = scale * (np.abs(q[:, h]) @ np.abs(k.T))
        s = np.where(seen, s, -np.inf)
        top = s.max(axis=1, initial=-np.inf, keepdims=True)
        p = np.exp(s - np.where(top == -np.inf, 0, top))
        p = np.where(seen, p, 0.0)
        total = p.sum(axis=1, keepdims=True)
        w = p / np.where(total == 0, 1.0, total)
        live = seen.any(axis=0)
        v = np.where(live[:, None], v, 0.0)
        out[:, h] = w @ v
        spread = w @ np.abs(v)
        # hd products and sums and the multiplication by the scale, on the exponent, above and below the line; the exponential itself (2^-22), and
        # sums over the keys
        e = 2 * ((hd + 4) * HALF["f32"] * np.where(seen, size, 0.0).max(axis=1, initial=0.0, keepdims=True) + 2.0 ** -22 +
                 (s.shape[1] / 8 + 16) * HALF["f32"])
        off = (HALF["bf16"] + e) * spread
        bound[:, h] = off + HALF["bf16"] * (np.abs(out[:, h]) + off) + 1e-38
    return out, bound

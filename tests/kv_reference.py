"""The paged cache operators from their definitions, in 64 bits on the host, sequence by sequence."""
import math

import numpy as np
import torch

STEPS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LIMITS = {torch.bfloat16: (-127, 125), torch.float16: (-23, 13)}


def half_step(dtype):
    """What one rounding to nearest may be off by, relative to the value."""
    return torch.finfo(dtype).eps / 2


def to_type(x, dtype):
    """64-bit values rounded to 32 bits and from there to `dtype`, as 64-bit values."""
    return torch.from_numpy(np.ascontiguousarray(x)).float().to(dtype).double().numpy()


def encode4(x, dtype):
    """Codes (0..15) and scale bytes of 64-bit values [..., 32 n] that are values of `dtype`."""
    low, high = LIMITS[dtype]
    b = x.reshape(-1, 32)
    codes, scales = np.zeros(b.shape, np.uint8), np.zeros(b.shape[0], np.uint8)
    for i, v in enumerate(b):
        if not np.isfinite(v).all():
            scales[i] = 255
            continue
        top, power = np.abs(v).max(), low
        while power < high and top > 7 * 2.0 ** power:
            power += 1
        scales[i] = power + 127
        y = np.abs(v) / 2.0 ** power
        off = np.abs(y[:, None] - STEPS)
        best = off.min(1, keepdims=True)
        first = (off == best).argmax(1)                                  # of two that are as near, the even code
        second = 7 - (off == best)[:, ::-1].argmax(1)
        code = np.where(first % 2 == 0, first, second)
        codes[i] = code + 8 * np.signbit(v)
    return codes.reshape(x.shape), scales.reshape(x.shape[:-1] + (x.shape[-1] // 32,))


def decode4(codes, scales):
    value = STEPS[codes % 8] * np.where(codes >= 8, -1.0, 1.0)
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (value.reshape(scales.shape + (32,)) * scale[..., None]).reshape(codes.shape)


def page_values(pool, bits, page_tokens, heads, dim):
    """A pool's pages [pages, tokens, heads, dim] in 64 bits."""
    if bits == 16:
        return pool.cpu().double().numpy()
    raw = pool.cpu().numpy()
    n = page_tokens * heads * dim
    c = raw[:, :n // 2]
    codes = np.stack([c & 15, c >> 4], -1).reshape(-1, page_tokens, heads, dim)
    return decode4(codes, raw[:, n // 2:n // 2 + n // 32].reshape(-1, page_tokens, heads, dim // 32))


def norm_rotate(x, weight, eps, turn, rope_dim, pairs):
    """x [rows, heads, dim]; turn [rows, rope_dim] or None."""
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    if turn is None:
        return x
    half = rope_dim // 2
    cos, sin = turn[:, None, :half], turn[:, None, half:]
    at = (slice(0, rope_dim, 2), slice(1, rope_dim, 2)) if pairs else (slice(0, half), slice(half, rope_dim))
    a, b = x[..., at[0]], x[..., at[1]]
    y = x.copy()
    y[..., at[0]], y[..., at[1]] = a * cos - b * sin, b * cos + a * sin
    return y


def attend(q, k, v, scale, window, causal):
    """One sequence: q [rows, q_heads, dim], k and v [tokens, heads, dim] -> out, lse, and per row and head what bounds its
    error: sum of weights times |v|, and the largest sum of |q| |k| over the tokens that it sees."""
    rows, q_heads, dim = q.shape
    n, heads = k.shape[0], k.shape[1]
    out, lse = np.zeros((rows, q_heads, dim)), np.full((rows, q_heads), -math.inf)
    mass, size = np.zeros((rows, q_heads, dim)), np.zeros((rows, q_heads))
    for r in range(rows):
        hi = n - rows + r + 1 if causal else n
        lo = max(0, hi - window) if window else 0
        if hi <= lo:
            continue
        for h in range(q_heads):
            kk, vv = k[lo:hi, h // (q_heads // heads)], v[lo:hi, h // (q_heads // heads)]
            s = kk @ q[r, h] * scale
            top = s.max()
            if top == -math.inf:
                continue
            w = np.exp(s - top)
            lse[r, h] = top + math.log(w.sum()) if not np.isnan(w.sum()) else math.nan
            w = w / w.sum()
            out[r, h] = w @ vv
            mass[r, h] = w @ np.abs(vv)
            size[r, h] = scale * (np.abs(kk) @ np.abs(q[r, h])).max()
    return out, lse, mass, size


def attend_bounds(out, mass, size, tokens, dim, dtype):
    """How far outputs and logsumexps computed in 32 bits may be off.  A score's sum of `dim` products is off by (dim + 8) 2^-24
    of its absolute terms, weights by that (twice, with the maximum's) and the few roundings of their exponential; a sum of
    weights by 2^-24 a token; weights are rounded to the type once, and so is the result (to nothing finer than its least step)."""
    u, e = half_step(dtype), 2.0 ** -24
    score = (dim + 8) * e * size
    weight = 2 * score + (tokens + 64) * e
    info = torch.finfo(dtype)
    return (u + 2 * weight[..., None]) * mass * (1 + u) + u * np.abs(out) + info.tiny * info.eps, 2 * score + (tokens + 64) * e

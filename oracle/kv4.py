"""A cache of keys and values in 4 bits, and attention over it, in float64.

The format (groups of min(head_dim, 64) channels; steps in float32): scale = bf16((hi - lo) * (1 / 15)), low = bf16(lo); a value is the
whole number in [0, 15] nearest to (value - low) / scale (even one of two, 0 where scale is 0) and stands for low + scale * number.
"""
import numpy as np


def bf16(x):
    """float32 -> the nearest bfloat16 (even one of two), as float32."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    r = (b + np.uint32(0x7FFF) + ((b >> np.uint32(16)) & np.uint32(1))) & np.uint32(0xFFFF0000)
    return np.where(np.isnan(x), np.float32(np.nan), r.view(np.float32))


def quantise(x):
    """x float32 [..., head_dim] -> (numbers int64 [..., groups, channels], scale, low float64 [..., groups]); NaN scale and low for a group
    that holds an infinity or a NaN or whose range is beyond float32."""
    x = np.asarray(x, dtype=np.float32)
    group = min(x.shape[-1], 64)
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // group, group))
    with np.errstate(all="ignore"):
        lo, hi = g.min(-1), g.max(-1)
        range15 = (hi - lo) * (np.float32(1) / np.float32(15))
        good = np.isfinite(g).all(-1) & np.isfinite(range15)
        scale = np.where(good, bf16(range15), np.float32(np.nan)).astype(np.float64)
        low = np.where(good, bf16(lo), np.float32(np.nan)).astype(np.float64)
        n = np.rint((g.astype(np.float64) - low[..., None]) / scale[..., None])
    n = np.where(scale[..., None] > 0, np.clip(n, 0, 15), 0)
    return n.astype(np.int64), scale, low


def values(n, scale, low):
    """What the numbers stand for, float64 [..., head_dim]."""
    v = n * scale[..., None] + low[..., None]
    return v.reshape(v.shape[:-2] + (v.shape[-2] * v.shape[-1],))


def attention(q, k, v, n_rows, scale):
    """One sequence: q [n_rows, heads, head_dim], k and v = quantise(...) of its tokens [tokens, kv_heads, ..].  Row i sees the positions
    0 .. tokens - n_rows + i.  Returns (out float64 [n_rows, heads, head_dim], bound of what a computation in float32 with weights rounded
    to bf16 and a bf16 result may be off).

    The bound.  A weight times its scale is rounded to bf16 (2^-8 relative) and meets the whole value, number and low; the result is
    rounded (2^-8).
    In float32 (2^-24 an operation): a score is a sum of head_dim products q (16 + c) scale and of (low - 16 scale) sum q, in at most
    head_dim + 16 operations; an error d of the scores changes each weight by a factor within exp(+-d), so the result by 2 d sum w |v|;
    exponentials are good to 2^-21 with the rounding of their arguments; and the sums over the tokens take at most tokens / 8 + 64 operations on
    terms (16 + c) scale and low - 16 scale."""
    tokens, heads, share = k[0].shape[0], q.shape[1], q.shape[1] // k[0].shape[1]
    kv, vv = values(*k), values(*v)
    hd = q.shape[2]
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    reach = (np.abs(v[1])[..., None] * (32 + v[0]) + np.abs(v[2])[..., None]).reshape(vv.shape)
    for i in range(n_rows):
        n = tokens - n_rows + i + 1
        if n <= 0:
            continue
        for h in range(heads):
            g = h // share
            x = scale * (kv[:n, g] @ q[i, h])
            size = (np.abs(q[i, h]).reshape(1, -1, min(hd, 64)).sum(-1) * (47 * np.abs(k[1][:n, g]) + np.abs(k[2][:n, g]))).sum(-1)
            d = (abs(scale) * size * (hd + 16) * 2.0 ** -24).max() + 2.0 ** -21 * (1 + np.abs(x - x.max()).max() / 8)
            w = np.exp(x - x.max())
            w /= w.sum()
            out[i, h] = w @ vv[:n, g]
            bound[i, h] = 2.0 ** -8 * np.abs(out[i, h]) + 2.0 ** -8 * (w @ np.abs(vv[:n, g])) + 2 * d * (w @ np.abs(vv[:n, g])) + \
                (tokens / 8 + 64) * 2.0 ** -24 * (w @ reach[:n, g])
            bound[i, h] *= 1.02                             # products of the above
    return out, bound


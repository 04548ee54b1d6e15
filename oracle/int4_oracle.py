"""Float64 numpy reference of the verify step in 4 bits (test infrastructure).

Written from the definitions of include/spade.h alone; shares no code with the CUDA path or with
the package's set-up code.  Caches are given as pools with their block table; a sequence's slots
are gathered here one page at a time.
"""
from __future__ import annotations

import numpy as np

ORDER = (0, 2, 4, 6, 1, 3, 5, 7)  # number held by field p (bits 4p .. 4p + 3) of a word


def codes_of(packed):
    """Bytes [..., n / 2] -> codes [..., n]."""
    packed = np.ascontiguousarray(packed)
    words = packed.view("<u4")
    out = np.zeros(words.shape[:-1] + (words.shape[-1] * 8,), dtype=np.int64)
    for p, number in enumerate(ORDER):
        out[..., number::8] = (words >> np.uint32(4 * p)) & np.uint32(15)
    return out


def values(packed, params):
    """What codes and (scale, zero) pairs stand for, float64 [..., n]."""
    c = codes_of(packed).astype(np.float64)
    group = c.shape[-1] // params.shape[-2]
    s = np.repeat(params[..., 0].astype(np.float64), group, axis=-1)
    z = np.repeat(params[..., 1].astype(np.float64), group, axis=-1)
    with np.errstate(invalid="ignore"):
        return s * (c - z)


def linear(x, packed, params, residual=None):
    """(y, sum of |x w|) of y = x W^T (+ residual)."""
    w = values(packed, params)
    y = x.astype(np.float64) @ w.T
    mass = np.abs(x).astype(np.float64) @ np.abs(w).T
    return (y if residual is None else y + residual), mass


def slots(pool, table_row, first, count):
    """[count, Hkv, ...] of a pool [pages, Hkv, page, ...]."""
    page = pool.shape[2]
    return np.stack([pool[table_row[s // page], :, s % page] for s in range(first, first + count)])


def attention(q, pools, table, ctx, k, cu):
    """(out, lse, mass, score mass): rows [R, Hq, D]; mass = sum_s p |v|, score mass = max_s sum_d |q k| / sqrt(D)."""
    R, Hq, D = q.shape
    out, mass = np.zeros((R, Hq, D)), np.zeros((R, Hq, D))
    lse, smass = np.zeros((R, Hq)), np.zeros((R, Hq))
    kc, kp, vc, vp = pools
    G = Hq // kc.shape[1]
    for b in range(len(ctx)):
        n = int(ctx[b] + k[b] + 1)
        K = values(slots(kc, table[b], 0, n), slots(kp, table[b], 0, n))
        V = values(slots(vc, table[b], 0, n), slots(vp, table[b], 0, n))
        for i in range(int(k[b]) + 1):
            seen = int(ctx[b]) + i + 1
            for h in range(Hq):
                r = int(cu[b]) + i
                qv = q[r, h].astype(np.float64)
                with np.errstate(invalid="ignore"):
                    s = K[:seen, h // G] @ qv / np.sqrt(D)
                    smass[r, h] = (np.abs(K[:seen, h // G]) @ np.abs(qv)).max() / np.sqrt(D)
                    top = s.max()
                    p = np.exp(s - top)
                    total = p.sum()
                    p /= total
                    out[r, h] = p @ V[:seen, h // G]
                    mass[r, h] = p @ np.abs(V[:seen, h // G])
                    lse[r, h] = top + np.log(total)
    return out, lse, mass, smass


def turned(x, weight, turn, eps):
    """Heads x [R, H, D] normed (weight None: not) and rotated by turn [R, D / 2, 2]; and the size of what is summed."""
    x = x.astype(np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight.astype(np.float64)
    half = x.shape[-1] // 2
    z = (x[..., :half] + 1j * x[..., half:]) * (turn[..., 0].astype(np.float64) + 1j * turn[..., 1])[:, None]
    size = np.hypot(x[..., :half], x[..., half:])
    return np.concatenate([z.real, z.imag], -1), np.concatenate([size, size], -1)


def check_quantised(x, err, packed, params):
    """Whether (codes, pairs) are a rounding of numbers x [..., D], each known to within err: the pair's scale is
    fp16(span / 15) for a span within the error, zero and codes are the nearest whole numbers but for ties that
    the error reaches; a group with a number that is not finite has the scale NaN, and no other one has.  Returns the
    number of violations."""
    c = codes_of(packed).reshape(x.shape[:-1] + (-1, 64)).astype(np.float64)
    x = x.reshape(c.shape)
    finite = np.isfinite(x).all(-1)
    x = np.where(finite[..., None], x, 0.0)
    e = np.where(finite, err.reshape(c.shape).max(-1), 0.0)
    s, z = params[..., 0].astype(np.float64), params[..., 1].astype(np.float64)
    lo, hi = np.minimum(x.min(-1), 0), np.maximum(x.max(-1), 0)
    span, tol = (hi - lo) / 15, 2 * e / 15 + 2.0 ** -22 * (hi - lo)
    low = np.minimum(span - tol, 4364.0).clip(min=0).astype(np.float16).astype(np.float64)
    high = np.minimum(span + tol, 4364.0).astype(np.float16).astype(np.float64)
    bad = ~((s >= low) & (s <= high))
    live = s > 0
    safe = np.where(live, s, 1.0)
    slack = e / safe + 2.0 ** -20 * (1 + np.abs(lo / safe))
    bad |= live & ~(np.abs(z - np.clip(-lo / safe, 0, 15)) <= 0.5 + slack)
    bad |= ~((z == np.round(z)) & (z >= 0) & (z <= 15)) | (~live & (z != 0))
    at = x / safe[..., None] + z[..., None]
    want = np.clip(at, 0, 15)
    off = ~(np.abs(c - want) <= 0.5 + slack[..., None])
    off = np.where(live[..., None], off, c != 0)
    bad = np.where(finite, bad, ~np.isnan(s))
    return int(bad.sum() + (off & finite[..., None]).sum())

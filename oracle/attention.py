"""The attention half of a layer in fp64 on the CPU (test infrastructure only):
4-bit weights, the 4-bit paged cache, rotation, attention and block norms, read
from the formats that include/moe_offload.h states.
"""
from __future__ import annotations

import numpy as np

GROUP = 64       # columns of a weight group
KV_GROUP = 32    # dimensions of a cache group
STEPS = np.array([(8 + k % 8) * 2.0 ** (k // 8 - 24) for k in range(255)])


# -- 4-bit weights ------------------------------------------------------------

def q4_dequantize(buf: np.ndarray, n: int, k: int) -> np.ndarray:
    """fp64 [n x k] from one stored matrix (uint8)."""
    buf = np.asarray(buf, dtype=np.uint8)
    assert k % GROUP == 0 and buf.size == n * k // 2 + n * k // GROUP * 3
    codes = buf[:n * k // 2].reshape(n, k // 2)
    scale = buf[n * k // 2:n * k // 2 + n * k // 32].copy().view("<f2").astype(np.float64).reshape(n, k // GROUP)
    zero = buf[n * k // 2 + n * k // 32:].astype(np.float64).reshape(n, k // GROUP) / 16
    q = np.empty((n, k))
    q[:, 0::2], q[:, 1::2] = codes & 15, codes >> 4
    return (q - np.repeat(zero, GROUP, 1)) * np.repeat(scale, GROUP, 1)


# -- cache entries ------------------------------------------------------------

def kv4_quantize(x: np.ndarray):
    """Codes [..., D] and metas [..., D/32] of x [..., D], in x's precision
    (fp32 gives the library's bits)."""
    x = np.asarray(x)
    one = x.dtype.type
    g = x.reshape(*x.shape[:-1], -1, KV_GROUP)
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[..., None], g, one(0))
    lo, hi = np.minimum(g.min(-1), one(0)), np.maximum(g.max(-1), one(0))
    steps = STEPS.astype(x.dtype)
    k = np.minimum(np.searchsorted(one(15) * steps, hi - lo), 254)  # 15 * step is exact
    s = steps[k]
    with np.errstate(over="ignore"):
        z = np.clip(np.rint(-lo / s), 0, 15).astype(x.dtype)
        q = np.clip(np.rint(g / s[..., None]) + z[..., None], 0, 15)
    q = np.where(fine[..., None], q, 0)
    k, z = np.where(fine, k, 255), np.where(fine, z, 0)
    return q.reshape(x.shape).astype(np.uint8), (k << 8 | z.astype(np.int64)).astype(np.uint16)


def kv4_values(codes: np.ndarray, metas: np.ndarray) -> np.ndarray:
    k = (metas >> 8).astype(np.int64)
    s = np.where(k == 255, np.nan, STEPS[np.minimum(k, 254)])
    q = codes.astype(np.float64).reshape(*codes.shape[:-1], -1, KV_GROUP)
    return ((q - (metas & 255).astype(np.float64)[..., None]) * s[..., None]).reshape(codes.shape)


def record(kq, km, vq, vm) -> np.ndarray:
    """One record's bytes from codes [P, D] and metas [P, D/32] of keys and values."""
    P, D = kq.shape
    vq = vq.reshape(P // 4, 4, D // 8, 8).transpose(0, 2, 1, 3)
    vm = vm.reshape(P // 4, 4, D // KV_GROUP).transpose(0, 2, 1)
    nib = [np.ascontiguousarray(c).reshape(-1) for c in (kq, vq)]
    return np.concatenate([c[0::2] | c[1::2] << 4 for c in nib]
                          + [np.ascontiguousarray(m).astype("<u2").reshape(-1).view(np.uint8) for m in (km, vm)])


def unpack_record(rec: np.ndarray, P: int, D: int):
    """(key codes, key metas, value codes, value metas) of one record."""
    def nibbles(c):
        out = np.empty(2 * c.size, dtype=np.uint8)
        out[0::2], out[1::2] = c & 15, c >> 4
        return out
    h, m = P * D // 2, P * D // 16
    kq = nibbles(rec[:h]).reshape(P, D)
    vq = nibbles(rec[h:2 * h]).reshape(P // 4, D // 8, 4, 8).transpose(0, 2, 1, 3).reshape(P, D)
    km = rec[2 * h:2 * h + m].copy().view("<u2").reshape(P, D // KV_GROUP)
    vm = rec[2 * h + m:].copy().view("<u2").reshape(P // 4, D // KV_GROUP, 4).transpose(0, 2, 1).reshape(P, D // KV_GROUP)
    return kq, km, vq, vm


def gather(pool: np.ndarray, pages, length: int, P: int, D: int):
    """Keys and values [heads, length, D] in fp64 of a sequence over `pages`;
    held [length] is False where no page is named."""
    heads = pool.shape[1]
    k, v = np.zeros((2, heads, length, D))
    held = np.zeros(length, dtype=bool)
    for c, page in enumerate(pages):
        lo, hi = c * P, min((c + 1) * P, length)
        if lo >= hi:
            break
        if not 0 <= page < pool.shape[0]:
            continue
        held[lo:hi] = True
        for h in range(heads):
            kq, km, vq, vm = unpack_record(pool[page, h], P, D)
            k[h, lo:hi], v[h, lo:hi] = kv4_values(kq, km)[:hi - lo], kv4_values(vq, vm)[:hi - lo]
    return k, v, held


# -- the block ----------------------------------------------------------------

def rotate(x, cos, sin):
    """x [tokens, heads, D] turned by cos, sin [tokens, rot/2], in their precision."""
    half = cos.shape[1]
    out = np.array(x)
    a, b, c, s = x[..., :half], x[..., half:2 * half], cos[:, None], sin[:, None]
    out[..., :half], out[..., half:2 * half] = a * c - b * s, b * c + a * s
    return out


def attention(q, k, v, seen, scale: float):
    """o [n, D] of queries q [n, D] over k, v [m, D]; seen [n, m] bool."""
    out = np.zeros((q.shape[0], v.shape[1]))
    for i in range(q.shape[0]):
        at = np.flatnonzero(seen[i])
        if at.size:
            z = scale * (k[at] @ q[i])
            p = np.exp(z - z.max())
            out[i] = (p / p.sum()) @ v[at]
    return out


def norm_residual(h, y=None, gate=None, post=None, pre=None, residual_scale=1.0, eps=1e-5):
    def rms(t):
        return np.sqrt(np.mean(t * t, -1, keepdims=True) + eps)
    h = np.asarray(h, dtype=np.float64) * residual_scale
    if y is not None:
        y = np.asarray(y, dtype=np.float64)
        if post is not None:
            y = y / rms(y) * post
        h = h + (1.0 if gate is None else gate) * y
    return h, h / rms(h) * (1.0 if pre is None else pre)

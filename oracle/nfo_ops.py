"""fp64 oracle of the operators a step is composed from: group normalisation, linear layers, dropout, the 8-bit cache.

Plain numpy in double precision, one function per formula, no code shared with the library.  Where an operator's definition itself
rounds (the quantiser's fp32 scale and reciprocal, the dropout factor, the ReLU mask of group normalisation) the rounding is written out.
"""
import math

import numpy as np

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def act(z, kind):
    if kind == "relu":
        return np.where(z < 0, 0.0, z)
    if kind == "silu":
        with np.errstate(over="ignore"):
            return z / (1.0 + np.exp(-z))
    if kind == "gelu":
        return 0.5 * z * _erfc(-z / math.sqrt(2.0))
    return z


def act_grad(z, kind):
    if kind == "relu":
        return (z > 0).astype(np.float64)
    if kind == "silu":
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if kind == "gelu":
        return 0.5 * _erfc(-z / math.sqrt(2.0)) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return np.ones_like(z)


def group_stats(x, groups, eps):
    """x [N, P, C] -> mean, rstd [N, groups]."""
    N, P, C = x.shape
    v = x.astype(np.float64).reshape(N, P, groups, C // groups)
    mean = v.mean(axis=(1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    return mean, 1.0 / np.sqrt(var + eps)


def _per_channel(t, C):
    return np.repeat(t, C // t.shape[1], axis=1)[:, None, :]


def group_norm(x, gamma, beta, groups, eps, kind):
    """(y, mean, rstd, z)"""
    C = x.shape[2]
    mean, rstd = group_stats(x, groups, eps)
    z = gamma * ((x - _per_channel(mean, C)) * _per_channel(rstd, C)) + beta
    return act(z, kind), mean, rstd, z


def relu_mask_f32(x, gamma, beta, mean, rstd):
    """The sign decision as the operator defines it: subtraction, product, product, sum, each rounded to fp32."""
    f = np.float32
    C = x.shape[2]
    xh = (x.astype(f) - _per_channel(mean.astype(f), C)) * _per_channel(rstd.astype(f), C)
    return (xh * gamma.astype(f) + beta.astype(f)) > 0


def group_norm_grad(x, dy, gamma, beta, mean, rstd, kind):
    """(dx, dgamma, dbeta, per-channel sums of |dz xh| and |dz|) at the given statistics."""
    N, P, C = x.shape
    G = mean.shape[1]
    mu, rs = _per_channel(mean.astype(np.float64), C), _per_channel(rstd.astype(np.float64), C)
    xh = (x - mu) * rs
    dz = dy * (relu_mask_f32(x, gamma, beta, mean, rstd) if kind == "relu" else act_grad(gamma * xh + beta, kind))
    e = (dz * gamma).reshape(N, P, G, C // G)
    m1 = e.mean(axis=(1, 3))
    m2 = (e * xh.reshape(e.shape)).mean(axis=(1, 3))
    dx = rs * (dz * gamma - _per_channel(m1, C) - xh * _per_channel(m2, C))
    return dx, (dz * xh).sum(axis=(0, 1)), dz.sum(axis=(0, 1)), np.abs(dz * xh).sum(axis=(0, 1)), np.abs(dz).sum(axis=(0, 1))


def linear(x, w, bias, residual, kind):
    """(y, z)"""
    z = x.astype(np.float64) @ w.astype(np.float64).T
    if bias is not None:
        z = z + bias
    if residual is not None:
        z = z + residual
    return act(z, kind), z


def philox(seed, offset, count):
    """The words of the first `count` blocks of Philox4x32-10 (Salmon et al., 2011), key = seed, counter = (block, offset)."""
    out = np.empty((count, 4), dtype=np.uint32)
    M = 0xFFFFFFFF
    for i in range(count):
        c = [i & M, i >> 32, offset & M, (offset >> 32) & M]
        k = [seed & M, (seed >> 32) & M]
        for _ in range(10):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(b >> 32) ^ c[1] ^ k[0], b & M, (a >> 32) ^ c[3] ^ k[1], a & M]
            k = [(k[0] + 0x9E3779B9) & M, (k[1] + 0xBB67AE85) & M]
        out[i] = c
    return out


def dropout(x32, p, seed, offset):
    """x32 float32 -> float32, before the rounding to the storage type."""
    n = x32.size
    u = philox(seed, offset, (n + 3) // 4).reshape(-1)[:n].astype(np.uint64)
    p = float(np.float32(p))
    scale = np.float32(1.0 / (1.0 - p))
    with np.errstate(invalid="ignore", over="ignore"):
        return np.where(u >= int(p * 4294967296.0), x32.reshape(-1) * scale, np.float32(0)).reshape(x32.shape)


def e4m3_values():
    """The value of every e4m3 code: sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7f and 0xff are NaN."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v[c] = (m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)
        if e == 15 and m == 7:
            v[c] = np.nan
        if c & 128:
            v[c] = -v[c]
    return v


def _e4m3_code(q):
    """Nearest code, ties to the even mantissa, magnitudes above 448 at 448."""
    pos = e4m3_values()[:127]
    a = np.minimum(np.abs(q.astype(np.float64)), 448.0)
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return (np.where(up, hi, lo) | np.where(np.signbit(q), 128, 0)).astype(np.uint8)


def quantize(x, fmt, group):
    """x float32 [rows, E] -> (codes uint8, scales float32); a group with a non-finite value has a NaN for a scale (codes of no meaning)."""
    f = np.float32
    rows, E = x.shape
    n = -(-E // group)
    v = np.zeros((rows, n * group), dtype=f)
    v[:, :E] = x
    v = v.reshape(rows, n, group)
    bad = ~np.isfinite(v).all(axis=2)
    top = f(127 if fmt == "int8" else 448)
    a = np.maximum(np.abs(np.where(bad[:, :, None], f(1), v)).max(axis=2), f(2.0 ** -100))
    q = np.where(bad[:, :, None], f(0), v) * (top / a)[:, :, None]
    if fmt == "int8":
        codes = np.clip(np.rint(q), -127, 127).astype(np.int8).view(np.uint8)
    else:
        codes = _e4m3_code(q)
    return codes.reshape(rows, n * group)[:, :E], np.where(bad, f(np.nan), a / top).astype(f)


def dequantize(codes, scales, fmt, group):
    """float32 values before the rounding to the storage type."""
    E = codes.shape[1]
    v = codes.view(np.int8).astype(np.float32) if fmt == "int8" else e4m3_values()[codes].astype(np.float32)
    return v * np.repeat(scales, group, axis=1)[:, :E]

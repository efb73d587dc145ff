"""Oracle: projection by weights of 4 bits with a scale and a zero point per group.

Test infrastructure only (see the package docstring).  Float64 and Python integers.

* ``quantise``  codes, scales and zero points of a matrix: of a group's values and 0 the range
                [lo, hi] goes to 0..15;
* ``pack``      bytes of the packed layout, one code after the other; ``unpack`` reads them back;
* ``apply``     residual + bias + x W^T with W = s (q - z).
"""
from __future__ import annotations

import numpy as np


def bf16(v):
    """Nearest bf16 value of fp32 values (ties to even, subnormal ones too), as float64."""
    u = np.atleast_1d(np.asarray(v, np.float32)).view(np.uint32).astype(np.int64)
    u = np.where(np.isfinite(v), (u + 0x7fff + (u >> 16 & 1)) & 0xffff0000, u)
    return u.astype(np.uint32).view(np.float32).astype(np.float64).reshape(np.shape(v))


def padded(K):
    return -(-K // 128) * 128


def quantise(w, group):
    """w [N, K] of bf16 values as float64.  Returns (q [N, K], s [N, groups], z [N, groups])."""
    N, K = w.shape
    groups = padded(K) // group
    q, s, z = np.zeros((N, K), np.int64), np.zeros((N, groups)), np.zeros((N, groups))
    for n in range(N):
        for g in range(-(-K // group)):
            v = w[n, g * group:(g + 1) * group]
            if not np.isfinite(v).all():
                s[n, g] = np.nan
                continue
            lo, hi = min(0.0, v.min()), max(0.0, v.max())
            s[n, g] = bf16(np.float32((hi - lo) / 15))
            if s[n, g] > 0:
                z[n, g] = np.clip(np.rint(-lo / s[n, g]) + 0.0, 0, 15)
                q[n, g * group:(g + 1) * group] = np.clip(np.rint(v / s[n, g]) + z[n, g], 0, 15)
    return q, s, z


def _bf16_bits(v):
    """Patterns of bf16 values; one for every NaN."""
    return np.where(np.isnan(v), np.uint32(0x7fc0), np.asarray(v, np.float32).view(np.uint32) >> 16)


def pack(q, s, z):
    """uint8 bytes; s and z are bf16 values."""
    N, K = q.shape
    Kp, groups = padded(K), s.shape[1]
    codes = np.zeros((N, Kp // 8), np.uint32)       # 32-bit words
    for k in range(K):
        block, j, a, e = k // 128, k % 128 // 32, k % 32 // 8, k % 8
        codes[:, block * 16 + 4 * a + j] |= (q[:, k] << (4 * (e // 2) + 16 * (e % 2))).astype(np.uint32)
    words = (_bf16_bits(s) << 16 | _bf16_bits(z)).T.copy()
    return np.concatenate([codes.reshape(-1).view(np.uint8), words.reshape(-1).view(np.uint8)])


def unpack(data, N, K, group):
    Kp = padded(K)
    codes = data[:N * Kp // 2].view(np.uint32).reshape(N, Kp // 8)
    words = data[N * Kp // 2:].view(np.uint32).reshape(Kp // group, N)
    q = np.zeros((N, K), np.int64)
    for k in range(K):
        block, j, a, e = k // 128, k % 128 // 32, k % 32 // 8, k % 8
        q[:, k] = codes[:, block * 16 + 4 * a + j] >> (4 * (e // 2) + 16 * (e % 2)) & 15
    s = (words & 0xffff0000).astype(np.uint32).view(np.float32).astype(np.float64).T
    z = (words << 16).astype(np.uint32).view(np.float32).astype(np.float64).T
    return q, s, z


def apply(x, q, s, z, group, bias=None, residual=None):
    """x [T, K] float64.  Returns (y, size): size = sum |s| (32 + q + |z|) |x|, what the 32-bit sums of
    products with 16 + q and 16 + z go through."""
    K = q.shape[1]
    g = np.arange(K) // group
    y = x @ (s[:, g] * (q - z[:, g])).T
    size = np.abs(x) @ (np.abs(s[:, g]) * (32 + q + np.abs(z[:, g]))).T
    if bias is not None:
        y = y + bias
        size = size + np.abs(bias)
    if residual is not None:
        y = y + residual
        size = size + np.abs(residual)
    return y, size

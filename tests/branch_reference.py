"""The pointwise branch over rows in 64 bits, from its definitions, and how far the kernels may be off: rows in 8 bits,
root-mean-square norms, activations, matrix products.  Arrays are [rows][channels].
"""
import math

import numpy as np
import torch
from scipy.special import erfc, expit

from norm_reference import ROUNDOFF, TINY, TYPES, U, rounded  # noqa: F401

ACTS = ("none", "relu", "gelu", "silu")


def blocks(C):
    return (C + 31) // 32


def e4m3_table():
    """What the 256 codes stand for (OCP e4m3: exponent bias 7, subnormals, no infinities, 0x7f and 0xff NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = math.nan if e == 15 and m == 7 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = -v if c >= 128 else v
    return out


TABLE = e4m3_table()


def scale_byte(most):
    """The smallest s from 0 on with 448 * 2^(s - 127) >= most, from the definition in whole numbers."""
    s = 0
    while s < 254 and 448.0 * 2.0 ** (s - 127) < most:
        s += 1
    return 0 if most == 0 else s


def pack(v):
    """Binary32 values (numpy) -> (codes, scales): every code by the nearest of the 254 numbers, ties to the even code."""
    rows, C = v.shape
    B, W = blocks(C), (C + 127) // 128 * 4
    v64 = np.zeros((rows, 32 * B))
    v64[:, :C] = v
    scales = np.zeros((rows, W), np.uint8)
    codes = np.zeros((rows, 32 * B), np.uint8)
    up = TABLE[:127]  # 0 .. 448
    for r in range(rows):
        for b in range(B):
            part = v64[r, 32 * b:32 * b + 32]
            fine = np.isfinite(part)
            most = np.abs(part[fine]).max() if fine.any() else 0.0
            s = scale_byte(most)
            scales[r, b] = s
            x = np.abs(np.where(fine, part, 0.0)) / 2.0 ** (s - 127)
            hi = np.searchsorted(up, x).clip(0, 126)
            lo = (hi - 1).clip(0)
            dl, dh = x - up[lo], up[hi] - x
            code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
            code = np.where(fine, code, 127) | np.where(np.signbit(part), 128, 0)
            codes[r, 32 * b:32 * b + 32] = code
    return codes, scales


def unpack(codes, scales, C):
    by = 2.0 ** (scales[:, :blocks(C)].astype(np.float64) - 127)
    return (TABLE[codes] * np.repeat(by, 32, axis=1))[:, :C]


def same_codes(got, want):
    """Equal but for the sign of a NaN."""
    return bool(np.all((got == want) | (((got & 127) == 127) & ((want & 127) == 127))))


def half_step(v, scales):
    """How far the nearest code may be from each element of v: half a step of its binade, or of the smallest one, under its scale."""
    by = 2.0 ** (np.repeat(scales[:, :blocks(v.shape[1])].astype(np.float64), 32, axis=1)[:, :v.shape[1]] - 127)
    return np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10 * by)


def act(name, p):
    if name == "relu":
        return np.maximum(p, 0.0)
    if name == "gelu":
        return p * 0.5 * erfc(-p / math.sqrt(2))
    if name == "silu":
        return p * expit(p)
    return p.copy()


def slope(name, p):
    if name == "relu":
        return (p > 0).astype(np.float64)
    if name == "gelu":
        return 0.5 * erfc(-p / math.sqrt(2)) + p * np.exp(-p * p / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = expit(p)
        return s * (1 + p * (1 - s))
    return np.ones_like(p)


def act_error(name, p):
    """Of act(p), p exact, in binary32.  gelu: the tail's polynomial is off by 5e-7 of itself, its exponential by the rounding of its
    argument x^2 / 2 (three roundings, log2 e = 1.44) and 2 U more; past x = 0 the tail is taken off x, which adds a rounding.  silu: the argument of the
    exponential is rounded twice, the sum and the reciprocal once each (2 U for the hardware's), the product once."""
    if name == "gelu":
        tail = np.abs(p) * 0.5 * erfc(np.abs(p) / math.sqrt(2))
        return tail * (5e-7 + U * (3 * p * p / 2 * 1.45 + 8)) + U * np.abs(p) + 2.0 ** -126
    if name == "silu":
        y = np.abs(act("silu", p))
        return y * U * (2 * np.abs(p) + 8) + 2.0 ** -126 * (1 + np.abs(p))
    return np.zeros_like(p)


def slope_error(name, p):
    if name == "gelu":
        tail, density = 0.5 * erfc(np.abs(p) / math.sqrt(2)), np.exp(-p * p / 2) / math.sqrt(2 * math.pi)
        e = U * (3 * p * p / 2 * 1.45 + 8)
        return tail * (5e-7 + e) + np.abs(p) * density * e + 4 * U + 2.0 ** -126 * (1 + np.abs(p))
    if name == "silu":
        s = expit(p)
        return U * (2 * np.abs(p) + 12) * (s * (1 + np.abs(p))) + 2.0 ** -126 * (1 + np.abs(p))
    return np.zeros_like(p)


def stored(value, dtype):
    """One rounding to the storage type."""
    return 1.01 * ROUNDOFF[dtype] * np.abs(value) + TINY[dtype] / 2


# A sum over the C channels of a row goes through chains of at most 32 additions in a lane (four octets) for rows in registers, C / 1024 + 8 for
# any size, then a tree of ten and sixteen more; both are below C / 8 + 64, with the squares' own rounding.
def _chain(C):
    return C / 8 + 64


def rms(z, gamma, eps):
    """y and rstd in 64 bits."""
    rstd = 1.0 / np.sqrt((z * z).mean(axis=1, keepdims=True) + eps)
    return z * rstd * gamma, rstd[:, 0]


def rms_tolerance(z, gamma, eps, dtype):
    """Of y before its rounding, of y, of rstd: half the relative error of the sum, the square root's and the reciprocal's roundings."""
    y, rstd = rms(z, gamma, eps)
    e = (_chain(z.shape[1]) / 2 + 4) * U
    t = np.abs(y) * (e + 3 * U)
    return t, t + stored(y, dtype), rstd * e


def rms_backward(dy, dz, z, gamma, rstd):
    """dx, dgamma in 64 bits, with rstd as given."""
    r = rstd[:, None]
    xhat, g = z * r, dy * gamma
    return dz + r * (g - xhat * (g * xhat).mean(axis=1, keepdims=True)), (dy * xhat).sum(axis=0)


def rms_backward_tolerance(dy, dz, z, gamma, rstd, dtype, params):
    r = rstd[:, None]
    xhat, g = np.abs(z * r), np.abs(dy * gamma)
    dx, dgamma = rms_backward(dy, dz, z, gamma, rstd)
    s = (g * xhat).mean(axis=1, keepdims=True)
    t = r * (8 * U * (g + xhat * s) + (_chain(z.shape[1]) + 8) * U * xhat * s) + 4 * U * (np.abs(dx) + np.abs(dz))
    return t + stored(dx, dtype), rows_error(np.abs(dy) * xhat) + 2 * U * (np.abs(dy) * xhat).sum(axis=0) + stored(dgamma, params)


def rows_error(terms):
    """Of a sum over rows of terms: chains of at most rows / 4 + 16 in a lane or 4096 rows (parts are never more than 1024), then the parts'."""
    return (min(terms.shape[0], terms.shape[0] / 4 + 96)) * U * terms.sum(axis=0)


def matmul_error(a, b, packed):
    """Of sum_k a[m][k] b[n][k] (64-bit arrays [M][K], [N][K]) in binary32 on the matrix cores.  An instruction adds up 32 products (8-bit: 128) and its
    accumulator; whatever the order in it, at most one rounding (2 U: cut off) for each of them, and one for each instruction of the chain."""
    size = np.abs(a) @ np.abs(b).T
    step = 128 if packed else 32
    return (2 * step + 2 * math.ceil(a.shape[1] / step) + 64) * U * size

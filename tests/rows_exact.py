"""Norms over rows and rows in 8 bits in 64 bits, whole tensors at a time, for tests of what is stated to the last code: no rounding before the one that the definition has."""
import numpy as np

import branch_reference as ref

U = ref.U


def pack(v):
    """64-bit values -> (codes, scales) by the definition: the scale from the block's largest, the nearest of the 254 numbers, ties to the even code."""
    rows, C = v.shape
    B = ref.blocks(C)
    part = np.zeros((rows, B * 32))
    part[:, :C] = v
    part = part.reshape(rows, B, 32)
    m, e = np.frexp(np.abs(part).max(axis=2))  # m 2^e, 448 = 0.875 * 2^9
    s = np.where(m > 0, np.maximum(e - 9 + (m > 0.875) + 127, 0), 0)
    x = np.ldexp(np.abs(part), 127 - s[:, :, None])
    up = ref.TABLE[:127]
    hi = np.searchsorted(up, x).clip(0, 126)
    lo = (hi - 1).clip(0)
    dl, dh = x - up[lo], up[hi] - x
    codes = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi) | np.where(np.signbit(part), 128, 0)
    scales = np.zeros((rows, (C + 127) // 128 * 4), np.uint8)
    scales[:, :B] = s
    return codes.reshape(rows, B * 32).astype(np.uint8), scales


def norm(z, gamma, eps):
    """y and rstd."""
    rstd = 1.0 / np.sqrt((z * z).sum(axis=1) / z.shape[1] + eps)
    return z * rstd[:, None] * gamma, rstd


# The squares of binary32 numbers are exact in 64 bits, and so are sums of them to some C 2^-53; what is left is one rounding to binary32, a second word of rstd that is rounded
# itself (2^-48), and a product of that word and the first one's remainder with roundings of 2^-24 of some 2^-24: 2^-10 of a rounding holds all of that.  The smallest number beside it.
# A second word of rstd below 2^-126 is rounded to a multiple of 2^-149: 2^-150 off, and y = z rstd gamma by |z gamma| 2^-150 = |y| 2^-150 / rstd (nothing but for roots near 2^125).
def one_rounding(value, rstd=1.0):
    return (1 + 2.0 ** -10) * U * np.abs(value) + 2.0 ** -149 + np.abs(value) * 2.0 ** -150 / rstd

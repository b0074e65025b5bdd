"""Layer norm, dropout and the join of a residual branch in 64 bits, from their definitions, and how far the kernels may be off.

Arrays are [outer][C][inner].  Where the definition itself rounds (z of a join is stored in the tensors' type after a product and a
sum in binary32) the same roundings are made here, so that those outputs have one right value.
"""
import numpy as np
import torch

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# unit roundoff (half the distance of neighbours, relative) and the smallest distance of neighbours
ROUNDOFF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}
U = 2.0 ** -24


def philox(counter, key, rounds=10):
    """Philox-4x32 of the paper, in Python's own integers: four words of a four-word counter under a two-word key."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def words(n, seed, sequence, first=0):
    """The 32-bit words of elements first .. first + n - 1 (numpy; philox() above, vectorised)."""
    b0, b1 = first // 4, (first + n + 3) // 4
    e = np.arange(b0, b1, dtype=np.uint64)
    low, u32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    sequence, seed = sequence % 2 ** 64, seed % 2 ** 64
    c = [e & low, e >> u32, np.full_like(e, sequence & 0xFFFFFFFF), np.full_like(e, sequence >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> u32) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> u32) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, axis=1).reshape(-1)[first - 4 * b0:][:n]


def kept(shape, p, seed, sequence):
    n = int(np.prod(shape, dtype=np.int64))
    return (words(n, seed, sequence) >= np.uint64(round(p * 2.0 ** 32))).reshape(shape) if p < 1 else np.zeros(shape, bool)


def scale(p):
    return np.float32(1.0 / (1.0 - p)) if p < 1 else np.float32(0)


def dropout32(x, keep, p):
    """Dropout of binary32 values in binary32: what a join adds to the residual."""
    return np.where(keep, x * scale(p), np.float32(0)).astype(np.float32)


def rounded(v, dtype):
    """Binary32 (or 64-bit) numpy values -> the storage type, as a torch tensor on the CPU; one rounding from binary32."""
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).to(TYPES[dtype])


def norm(z, gamma, beta, eps):
    """y, mean, rstd in 64 bits."""
    mean = z.mean(axis=1, keepdims=True)
    rstd = 1.0 / np.sqrt(((z - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    return (z - mean) * rstd * gamma[:, None] + beta[:, None], mean[:, 0], rstd[:, 0]


def norm_backward(dy, z, gamma, mean, rstd):
    """The norm's gradients in 64 bits, with mean and rstd as given (what the call reads)."""
    mean, rstd = mean[:, None], rstd[:, None]
    xhat, g = (z - mean) * rstd, dy * gamma[:, None]
    dx = rstd * (g - g.mean(axis=1, keepdims=True) - xhat * (g * xhat).mean(axis=1, keepdims=True))
    return dx, (dy * xhat).sum(axis=(0, 2)), dy.sum(axis=(0, 2))


# How far a kernel may be off.  U is binary32's unit roundoff.  A sum over the C channels goes through chains of additions in binary32
# of at most C / 4 + 16 in all (4 lanes at least share a position, then a tree), a sum over the positions through at most
# positions / 256 + 64; a chain of n additions is off by at most n U times the sum of the terms' sizes (first order).
def _chain(C):
    return C / 4 + 16


def _stored(value, dtype):
    return 1.01 * ROUNDOFF[dtype] * np.abs(value) + TINY[dtype] / 2


def tolerances_forward(z, gamma, beta, eps, dtype):
    """Of y, mean and rstd.  The mean is corrected by the mean of the deviations from its first value, so it keeps its own rounding
    and the chain's share of deviations only; deviations are off by that and a rounding; the variance by its chain, rstd by half of it."""
    y, mean, rstd = norm(z, gamma, beta, eps)
    C = z.shape[1]
    size, spread = np.abs(z).max(axis=1), np.abs(z - mean[:, None]).mean(axis=1)
    first = _chain(C) * U * np.abs(z).mean(axis=1) + U * size  # the first mean's error: what the deviations carry more than spread
    t_mean = 2 * U * np.abs(mean) + 2 * U * size + 2 * _chain(C) * U * (spread + first)
    t_rstd = rstd * ((_chain(C) + 16) * U + 2 * (rstd * (first + U * size)) ** 2 + 4 * U * rstd * size)
    t_y = np.abs(gamma)[:, None] * (rstd[:, None] * (t_mean[:, None] + 2 * U * np.abs(z)) + np.abs(z - mean[:, None]) * t_rstd[:, None]) \
        + 4 * U * (np.abs(y - beta[:, None]) + np.abs(y))
    return t_y + _stored(y, dtype), t_mean, t_rstd


def tolerances_backward(dy, z, gamma, mean, rstd, dz, out, dtype, params, dgamma, dbeta):
    """Of the gradient of z (`out`, stored in the tensors' type), dgamma and dbeta (in the parameters')."""
    C, positions = z.shape[1], z.shape[0] * z.shape[2]
    m, r = mean[:, None], rstd[:, None]
    xhat, g = np.abs((z - m) * r), np.abs(dy * gamma[:, None])
    s1, s2 = g.mean(axis=1, keepdims=True), (g * xhat).mean(axis=1, keepdims=True)
    n = (_chain(C) + 16) * U
    t_dx = r * (8 * U * (g + s1 + xhat * s2) + n * (s1 + xhat * s2)) + 4 * U * (np.abs(out) + np.abs(dz))
    n = (positions / 256 + 64 + 8) * U
    t_dgamma, t_dbeta = n * (np.abs(dy) * xhat).sum(axis=(0, 2)), n * np.abs(dy).sum(axis=(0, 2))
    return t_dx + _stored(out, dtype), t_dgamma + _stored(dgamma, params), t_dbeta + _stored(dbeta, params)

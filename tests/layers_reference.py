"""What the operators of wide layers of experts are held to, in NumPy and 64 bits."""
import numpy as np


def held(x, matrix=False):
    """The values that x [.., a, b] stands for in 8 bits: blocks of 128 along b, 128 x 128 for matrices."""
    x = np.asarray(x, np.float64)
    out = np.empty_like(x)
    a, b = x.shape[-2:]
    for i in range(0, a, 128 if matrix else 1):
        rows = slice(i, min(a, i + 128) if matrix else i + 1)
        for j in range(0, b, 128):
            t = x[..., rows, j:j + 128]
            fine = np.isfinite(t)
            size = np.where(fine, np.abs(t), 0.0)
            top = size.max(axis=(-2, -1), keepdims=True)
            f, q = np.frexp(top)
            e = np.clip(np.where(top > 0, np.where(f > 0.875, q - 8, q - 9), -100), -100, 120)
            rel = size / np.exp2(e.astype(float))
            step = np.exp2(np.maximum(np.frexp(rel)[1] - 1, -6) - 3.0)
            # (2^128, which float32 has not, is 15/16 of it)
            v = np.minimum(np.rint(rel / step) * step * np.exp2(e.astype(float)), 15 * 2.0 ** 124)
            out[..., rows, j:j + 128] = np.where(fine, np.copysign(v, t), np.nan)
    return out


def silu(z):
    return z / (1 + np.exp(-z))


def dsilu(z):
    s = 1 / (1 + np.exp(-z))
    return s * (1 + z * (1 - s))


def groups(rng, n, k, E, empty=0.0, skip=()):
    """Experts [n, k] (-1: none), offsets and order as the grouping gives them."""
    ids = rng.integers(0, E, (n, k)).astype(np.int32)
    for e in skip:
        ids[ids == e] = (e + 1) % E
    ids[rng.random((n, k)) < empty] = -1
    key = np.where(ids.reshape(-1) >= 0, ids.reshape(-1), E)
    order = np.argsort(key, kind="stable").astype(np.int32)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(key, minlength=E + 1)[:E])]).astype(np.int32)
    return ids, offsets, order

"""fp64 oracle: the norm of all gradients, AdamW, its 8-bit states and its random bits.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).

AdamW with decoupled weight decay, t = step, g the scaled gradient:
  m <- b1 m + (1 - b1) g ;  v <- b2 v + (1 - b2) g^2
  p <- p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
8-bit states: e4m3 values (4 exponent bits of bias 7, 3 mantissa bits, fixed point below 2^-6) times a power of two per
block of 256, by which the block's largest magnitude lies in [128, 256).
"""
from __future__ import annotations

import numpy as np

F64 = np.float64
BLOCK = 256
CODES = np.arange(127)
GRID = np.where(CODES < 8, CODES * 2.0 ** -9, (1 + (CODES % 8) / 8) * 2.0 ** (CODES // 8 - 7.0))      # of the codes 0 .. 126


def mix(x):
    x = np.asarray(x, np.uint64) & np.uint64(0xffffffff)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x9E3779B1)) & np.uint64(0xffffffff)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xB504F333)) & np.uint64(0xffffffff)
    return x ^ (x >> np.uint64(16))


def random_bits(seed, step, tensor, n, first=0):
    """32 random bits of the elements first .. first + n - 1 of the tensor-th tensor of a call."""
    key = mix(int(mix(int(mix(seed)) + step)) + tensor)
    i = first + np.arange(n, dtype=np.uint64)
    high = i >> np.uint64(32)
    keys = np.where(high > 0, mix(key + high), key)
    return mix((i & np.uint64(0xffffffff)) ^ keys)


def step(p, m, v, g, t, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0):
    """Returns (p, m, v) after the step, in fp64."""
    p, m, v, g = (np.asarray(x, F64) for x in (p, m, v, g))
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p * (1 - lr * weight_decay) - lr / (1 - beta1 ** t) * m / (np.sqrt(v) / np.sqrt(1 - beta2 ** t) + eps)
    return p, m, v


def per_element(x, n):
    return np.repeat(x, BLOCK)[:n]


def exponents(x):
    """The power of two of every block (as the exponent), and how far the block's largest magnitude is from the next border, relatively."""
    x = np.abs(np.asarray(x, F64))
    a = np.pad(x, (0, -len(x) % BLOCK)).reshape(-1, BLOCK).max(1)
    with np.errstate(divide="ignore"):
        e = np.where(a > 0, np.floor(np.log2(a)) - 7, -126.0)
    e = np.maximum(e, -126.0)
    top = np.where(a > 0, a, 1.0) / 2.0 ** np.where(a > 0, e + 7, 0.0)      # in [1, 2)
    return e.astype(int), np.minimum(np.abs(top - 1), np.abs(2 - top))


def quantize(x, e, u, at_least_one=False):
    """Codes (without sign) of x / 2^e as e4m3 values, u in [0, 1) of a step added and the rest cut off, and how far (in steps) from the border to the
    other neighbour the value lay."""
    a = np.abs(np.asarray(x, F64)) / 2.0 ** per_element(e.astype(F64), len(x))
    low = np.searchsorted(GRID, a, side="right") - 1
    up = (a - GRID[low]) / (GRID[np.minimum(low + 1, 126)] - GRID[low]) + u
    code = low + (up >= 1)
    if at_least_one:
        code = np.where((a > 0) & (code == 0), 1, code)
    return code, np.minimum(np.abs(up - 1), np.minimum(np.abs(up), np.abs(2 - up)))


def norm(grads, max_norm=0.0):
    """(norm, factor that limits it)"""
    n = np.sqrt(sum(float((np.asarray(g, F64) ** 2).sum()) for g in grads))
    return n, 1.0 if max_norm == 0 or n <= max_norm else max_norm / n

"""The AdamW operators in 64 bits (numpy), with bounds on what fp32 arithmetic may differ by."""

import math

import numpy as np

U = 2.0 ** -24  # half a unit in the last place, relative
HYPER = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)


def matrix(shape):
    return (1, shape[0]) if len(shape) == 1 else (shape[0], math.prod(shape[1:]))


def blocking(shape):
    """(rows of a block, columns of a block, blocks) of a tensor, from the description."""
    n, m = matrix(shape)
    if m < 256:
        k = 256 // m
        return k, m, -(-n // k)
    nb = -(-m // 256)
    w = -(-m // nb)
    w += -w % 4
    return 1, w, n * nb


def block_of(shape):
    """The block of every element, row-major."""
    n, m = matrix(shape)
    k, w, _ = blocking(shape)
    i = np.arange(n * m)
    return (i // m) // k if m < 256 else (i // m) * -(-m // 256) + (i % m) // w


def step(t, p, m, v, g, c=1.0, decay=True, lr=3e-3, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1):
    """(p, m, v) after step t, all fp64."""
    b1, b2 = betas
    g = c * g
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    den = np.sqrt(v / (1 - b2 ** t)) + eps
    return p * (1 - (lr * weight_decay if decay else 0.0)) - lr / (1 - b1 ** t) * m / den, m, v


def bounds(t, p, m, v, g, dg, c=1.0, lr=3e-3, betas=(0.9, 0.99), eps=1e-6, **kw):
    """How far fp32 results may be from step()'s, for gradients known to within dg.

    m: the constants, two products, their sum and c g are each rounded: 6 U of the terms' magnitudes.
    v the same with g twice: 10 U.  p: of the update, m's 6 U, sqrt(v)'s half of 10 U and its own, three
    roundings of the denominator and three of the quotient and its factor (under 20 U in all); of p's
    own terms the decay factor, the product and the sum (4 U).  A gradient's own error moves the results
    by what step() says."""
    b1, b2 = betas
    size = b1 * np.abs(m) + (1 - b1) * np.abs(c * g)
    p1, m1, v1 = step(t, p, m, v, g, c, lr=lr, betas=betas, eps=eps, **kw)
    den = np.sqrt(v1 / (1 - b2 ** t)) + eps
    bp = U * (4 * np.abs(p) + 24 * lr / (1 - b1 ** t) * size / den)
    bm, bv = 6 * U * size, 10 * U * v1
    for s in (-1, 1):
        p2, m2, v2 = step(t, p, m, v, g + s * dg, c, lr=lr, betas=betas, eps=eps, **kw)
        bp, bm, bv = bp + np.abs(p2 - p1), bm + np.abs(m2 - m1), bv + np.abs(v2 - v1)
    tiny = 2.0 ** -140  # subnormal results
    return bp + tiny, bm + tiny, bv + tiny


# ---- the random rounding of 8-bit moments, from its description ----------------------------------------------

M32, M64 = 0xFFFFFFFF, 0xFFFFFFFFFFFFFFFF
GOLDEN = 0x9E3779B1


def _mix64(z):
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M64
    return z ^ (z >> 31)


def random_halves(seed, step, tensor, elements):
    """The 16 random bits of m and of sqrt(v) of these elements, as fractions of a rounding step."""
    k = ((_mix64((seed ^ _mix64(step)) & M64) >> 32) + tensor * GOLDEN) & M32
    k = ((k ^ (k >> 16)) * 0x85EBCA6B) & M32
    k = ((k ^ (k >> 13)) * 0xC2B2AE35) & M32
    k ^= k >> 16
    x = (np.asarray(elements, np.uint64) * np.uint64(GOLDEN) + np.uint64(k)) & np.uint64(M32)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x2C1B3C6D)) & np.uint64(M32)
    x ^= x >> np.uint64(12)
    return (x >> np.uint64(16)).astype(float) / 65536, (x & np.uint64(0xFFFF)).astype(float) / 65536


def code_values():
    """The values of the codes 0 to 126 (448)."""
    c = np.arange(127)
    return np.where(c < 8, c * 2.0 ** -9, (8 + c % 8) * 2.0 ** (c // 8 - 10.0))


def codes(y, dy, fraction, positive):
    """Codes of magnitudes y (of at most 448), rounded up where the dropped fraction of a step and `fraction` make
    one, and whether an error of dy in y leaves no doubt of it.  positive: a y > 0 is 2^-9 at least."""
    y = np.minimum(y, 448.0)
    if positive:
        y = np.where(y > 0, np.maximum(y, 2.0 ** -9), y)
    e = np.maximum(np.floor(np.log2(np.maximum(y, 2.0 ** -9))), -6.0)
    unit = 2.0 ** (e - 3)
    steps = y / unit + fraction
    # 20 bits of the fraction are kept, of numbers below 2^-6 perhaps fewer
    doubt = dy / unit + np.where(y < 2.0 ** -6, 2.0 ** -16, 2.0 ** -19)
    near = np.abs(steps - np.round(steps)) <= doubt
    # (the value's own power of two may be in doubt too, where it is within dy of one)
    near |= np.abs(y / 2.0 ** np.round(np.log2(np.maximum(y, 2.0 ** -12))) - 1) <= 2 * dy / np.maximum(y, 2.0 ** -12)
    return np.searchsorted(code_values(), np.floor(steps) * unit * (1 + 1e-9), side="right") - 1, ~near

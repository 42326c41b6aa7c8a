"""The optimizer step in 64 bits: AdamW with decoupled weight decay (Loshchilov, Hutter, ICLR'19) over the layers of
a flat buffer, and the 8-bit form of its moments.

Moments in 8 bits: a block of 128 elements from its layer's start shares an exponent byte x, the biased fp32
exponent of its largest magnitude (0 below the smallest normal number), one more where its mantissa exceeds 31/16.  Magnitudes lie on
a grid with 16 steps an octave over the octaves below 2^(x + 1 - 127), 7 of them for m and 15 for v, and on even steps, those
of the lowest octave, below.
"""
import numpy as np

from . import philox

BLOCK = 128
OCTAVES_M, OCTAVES_V = 7, 15


def decode(code, x, octaves):
    """Values of codes without sign under exponent bytes x (arrays of one shape)."""
    code, x = np.asarray(code, np.int64), np.asarray(x, np.int64)
    field, f = code >> 4, code & 15
    steps = np.where(field > 0, (16 + f) * 2.0 ** np.maximum(field - 1, 0), f)
    return steps * 2.0 ** (x - 127.0 - (octaves - 1) - 4)


def exponent(a):
    """Exponent byte of a block with these magnitudes (fp32 numbers held in any type)."""
    top = float(np.max(a))
    if top == 0.0:
        return 0
    mant, e = np.frexp(top)                       # top = mant 2^e, mant in [1/2, 1)
    e = int(e) - 1 + 127 + (2 * mant > 31 / 16)
    if e >= 1:
        return min(e, 255)
    return 1 if top > 15 / 16 * 2.0 ** -126 else 0


def grid(a, x, octaves):
    """The step of the grid at every magnitude of a block under exponent byte x."""
    a = np.asarray(a, np.float64)
    _, e = np.frexp(a)
    e = np.where(a > 0, e - 1, -10000)
    return 2.0 ** (np.maximum(e, x - 127 - (octaves - 1)) - 4)


def step(grads, p, m, v, t, lr, beta1, beta2, eps, decay, scale):
    """One layer's step: (p', m', v') in fp64 from arrays of any type; t counts from 1."""
    g = np.asarray(grads, np.float64) * scale
    p, m, v = (np.asarray(a, np.float64) for a in (p, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    update = m / (1 - beta1 ** t) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return p - lr * decay * p - lr * update, m, v


def clip(total, scale, max_norm):
    """Factor of the gradients under clipping, total = sum of their squares before `scale`."""
    return scale * min(1.0, max_norm / (scale * np.sqrt(total) + 1e-6)) if max_norm > 0 else scale


def rounded(a, x, octaves, u=None):
    """What 8 bits keep of a block's magnitudes under exponent byte x: to the nearest, ties to even, or, with numbers u
    in [0, 1), up where the part that is cut off reaches 1 - u of a step.  Grows with a."""
    h = grid(a, x, octaves)
    q = np.asarray(a, np.float64) / h
    return (np.rint(q) if u is None else np.floor(q + u)) * h


def halves(seed, t, layer, n):
    """The random numbers in [0, 1) of a layer's m and v in step t: centres of 2^16 intervals."""
    blk = np.arange((n + 3) // 4, dtype=np.uint64)
    same = np.ones(blk.size, np.uint64)
    w = np.stack(philox.philox4x32_10(blk, same * (t & 0xFFFFFFFF), same * layer, same * (1 + (t >> 32)),
                                      seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF), 1).reshape(-1)[:n]
    return ((w & 0xFFFF) + 0.5) / 65536, ((w >> 16) + 0.5) / 65536

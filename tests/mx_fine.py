"""Rows whose attention is wrong by much more than its bound unless probabilities keep 16
bits, and that bound.

The score of a key of class +1 is EPS' = log(1 + EPS), that of a key of class -1 is 0: weights
1 + EPS and 1. EPS = 0.9 2^-8 is less than half a step of bf16 there, so that rounded to bf16
once they are all 1. A key's values are its class times a sign of the dimension, and every two
neighbours are of different classes: with the right weights the result is EPS / 2 and a
rest of 1 / n at most, and the part that one rounding leaves out is EPS / 2, for n keys. A
second term for that rest has it to 2^-8, so a weight to 2^-16. Taken with other keys' values it
adds up to little, and with another dimension's to the wrong sign."""
import numpy as np

EPS = 0.9 * 2.0 ** -8
SCALE = float(np.log1p(EPS))          # of q k = 1


def rows(rng, n, hkv, d):
    """K and V [n][hkv][d], exact in codes of 4 and 8 bits; the dimensions' signs are the same
    in every call."""
    c = rng.choice([-1.0, 1.0], ((n + 1) // 2, 1, hkv))
    c = np.concatenate([c, -c], 1).reshape(-1, hkv)[:n]
    K = np.zeros((n, hkv, d))
    K[..., 0] = c > 0
    sign = np.random.default_rng(hkv * d).choice([-1.0, 1.0], (hkv, d // 2))
    return K, c[..., None] * np.stack([sign, -sign], -1).reshape(hkv, d)   # pairs differ


def queries(shape):
    """[..., d] with q k = 1 for a key of class +1."""
    q = np.zeros(shape)
    q[..., 0] = 1.0
    return q


def bound(ref, size, n, d):
    """As check_attend's for a bf16 result, but 2^-16 of a weight where that has 2^-8: its
    sum of products is one product, below 1, so ds = (d + 6) 2^-24 SCALE at most."""
    e = 2.0 ** -24
    w = 2 * ((d + 6) * e * SCALE + 4 * e) + (n + 16) * e
    return (w + 2.0 ** -16) * size + 2.0 ** -8 * np.abs(ref) + 1e-30

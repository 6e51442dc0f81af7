"""The bound of mx_fine tells two terms of a probability from one, and from a second term that
meets the wrong values: the mistakes are planted in a model of the arithmetic here."""
import numpy as np
import pytest

import mx_fine as F
from oracle import pages as OP


def _bf16(x):
    """To nearest, ties to even, of positive normal numbers."""
    u = x.astype(np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + (u >> 16 & 1)) >> 16 << 16
    return u.astype(np.uint32).view(np.float32).astype(np.float64)


def _model(K, V, rest, z):
    """One row's result [hkv][d] over all keys: P rounded once, and rest(P - that, V)."""
    p = np.exp(F.SCALE * K[..., 0]) * 2.0 ** -z                # [n][hkv]
    once = _bf16(p)
    o = (once[..., None] * V).sum(0) + rest(p - once, V)
    o /= p.sum(0)[:, None]
    return np.copysign(_bf16(np.abs(o) + 1e-38), o)


def _second(r, V):
    back = np.copysign(_bf16(np.abs(r) + 1e-38), r)
    return (back[..., None] * V).sum(0)


WRONG = {
    "no second term": lambda r, V: 0.0 * V[0],
    "the even dimension's values for the odd one's":
        lambda r, V: _second(r, V.reshape(len(V), -1, V.shape[2] // 2, 2)[..., ::-1].reshape(V.shape)),
    "values of eight keys further": lambda r, V: _second(r, np.roll(V, 8, 0)),
    "taken twice": lambda r, V: 2 * _second(r, V),
    "taken away": lambda r, V: -_second(r, V),
}


@pytest.mark.parametrize("n", [64, 300, 1100])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("z", [0, 1])
def test_two_terms_are_within_the_bound_and_others_are_not(n, d, z):
    rng = np.random.default_rng(n + d)
    K, V = F.rows(rng, n, 3, d)
    assert np.array_equal(OP.mx_values(K, 4), K) and np.array_equal(OP.mx_values(V, 4), V)
    assert np.array_equal(OP.mx_values(K, 8), K) and np.array_equal(OP.mx_values(V, 8), V)
    ref, _ = OP.attend(F.queries((1, 3, d)), K, V, F.SCALE)
    size, _ = OP.attend(F.queries((1, 3, d)), K, np.abs(V), F.SCALE)
    tol = F.bound(ref[0], size[0], n, d)
    assert np.all(np.abs(_model(K, V, _second, z) - ref[0]) <= tol)
    for name, rest in WRONG.items():
        off = np.abs(_model(K, V, rest, z) - ref[0]) > 2 * tol
        assert np.all(off.any(1)), name           # of every head

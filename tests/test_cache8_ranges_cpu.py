"""That the tolerances of test_gpu_cache8_ranges.py see the mistakes they are there for (planted in the results of
the 64-bit definition), and what the 8-bit cache's rows keep of their values, by the definition."""
import numpy as np
import pytest

from oracle import streaming as so
from test_gpu_cache8_ranges import BF, FP, _exact, _tolerance


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
def test_tolerances_see_planted_mistakes(d, dtype):
    """Rows of the smallest scale with the weight on them: zeros, or values a power of two off, in their place."""
    rng = np.random.default_rng(d)
    L = 900
    heavy = (np.arange(L) % 4 == 1)[:, None, None]
    q, k = np.zeros((1, 2, d)), np.zeros((L, 1, d))
    q[..., 0], k[..., 0] = 1, np.where(heavy[..., 0], 40.0, 0.0)
    small = rng.integers(8, 15, (L, 1, d)) * 2.0 ** rng.integers(0, 6, (L, 1, d)) * 2.0 ** -14
    v = np.where(heavy, small, _exact(1, L, d))
    want, _, tol = _tolerance(q, k, v, [L], 1.0, dtype)
    for wrong in (0.0, 0.5, 2.0):
        got = so.seq_attention(q, k, np.where(heavy, wrong * v, v), [L], 1.0)[0]
        assert np.all(np.abs(got - want) > tol)


@pytest.mark.parametrize("L", [900, 30011])
def test_tolerances_see_a_lost_tile_of_keys(L):
    """Unit normal q, k and v over many keys, one row of 128 channels: without 32 of the heavier keys some channel is past
    the tolerance."""
    d = 128
    q, k, v = np.random.default_rng(2).standard_normal((1, 1, d)), _exact(3, L, d), _exact(4, L, d)
    want, lse, tol = _tolerance(q, k, v, [L], 0.35, BF)
    p = np.exp(0.35 * (q[0, 0] @ k[:, 0].T) - lse[0, 0])
    p[np.argsort(p)[-64:-32]] = 0
    assert np.any(np.abs(p @ v[:, 0] - want[0, 0]) > tol[0, 0])


def test_what_a_row_keeps():
    """4 significant bits (half a step: 2^-4) down to 2^-13 of the row's largest or 2^-20, below that at most 2^-17 of the
    largest or 2^-24: rows of all sizes, those whose exponent is held at -14 among them, each with values far apart."""
    rng = np.random.default_rng(0)
    top = 2.0 ** rng.uniform(-26, 15.8, (4000, 1))
    x = top * 2.0 ** -rng.uniform(0, 24, (4000, 64)) * rng.choice([-1, 1], (4000, 64))
    m = np.abs(x).max(-1, keepdims=True)
    assert (m <= 57344).all() and (m < 2.0 ** -20).any()
    codes, scales = so.quantise_rows(x)
    off = np.abs(so.dequantise_rows(codes, scales) - x)
    whole = np.abs(x) >= np.maximum(2.0 ** -13 * m, 2.0 ** -20)
    assert whole.any() and np.all(off[whole] <= 2.0 ** -4 * np.abs(x[whole]))
    assert np.all(off <= np.where(whole, np.inf, np.maximum(2.0 ** -17 * m, 2.0 ** -24)))
    held = (scales == 113)[:, None]
    assert np.any(off > 2.0 ** -4 * np.abs(x), axis=-1, where=held).sum() > 100  # rows with fewer bits for some

"""The 8-bit cache's operators at the ends of their number ranges, against the 64-bit definitions (oracle.streaming):
factors of scores whose products leave 32 bits.

Tolerances of attention, where test_gpu_cache8.py allows more than a key can be off.  Weights are fp16 numbers,
the row's largest at least 2^7 (the reference point lies 2^7 below the running maximum, or lower), so a weight p
of a row's largest 1 is off by 2^-11 p, or where it is subnormal by 2^-25 2^-7 = 2^-32, and never by more than p:
min(max(2^-11 p, 2^-32), p) |v|.  What comes before a later maximum is scaled down with it.  The sum of weights is at
least 1, so this holds of the normed weights too.  On top: the sum of weights and the scores in 32 bits, 2^-11 of the
spread sum p |v|, and the output's rounding, eps |out| (fp16: 2^-25 at least)."""
import math

import numpy as np
import pytest
import torch

from oracle import streaming as so
from test_gpu_cache8 import BF, EPS, FP, Cache8, _cu, _dirty_ws, _f64, _randn, vpb
from test_gpu_cache8_edges import _ran

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    vpb.lib()


def _tolerance(q, k, v, lim, scale, dtype):
    """(out, lse, tolerance of out) of one sequence with one kv head."""
    out, lse, spread = so.seq_attention(q, k, v, lim, scale)
    off = np.zeros_like(out)
    for i, n in enumerate(lim):
        if n > 0:
            p = np.exp(scale * (q[i] @ k[:n, 0].T) - lse[i][:, None])
            off[i] = np.minimum(np.maximum(2.0 ** -11 * p, 2.0 ** -32), p) @ np.abs(v[:n, 0])
    return out, lse, EPS[dtype] * np.abs(out) + off + 2.0 ** -11 * spread + (2.0 ** -25 if dtype == FP else 0.0)


def _run(q, k, v, dtype, scale, kernel, block=1, page=32):
    """q [n][hq][d], k, v [L][1][d], exact in their types -> (out, lse) in 64 bits."""
    (n, hq, d), L = q.shape, k.shape[0]
    c = Cache8(1, [L], 1, d, page)
    c.dense[0] = [so.quantise_rows(x) for x in (k, v)]
    assert all(np.array_equal(so.dequantise_rows(*p), x) for p, x in zip(c.dense[0], (k, v)))
    c.write(0)
    dims = vpb.attn_dims(hq, 1, d, dtype=dtype, block=block, scale=scale)
    qt, ws = torch.from_numpy(q).to(dtype).cuda(), _dirty_ws(dims, n, 1)
    assert np.array_equal(_f64(qt), q, equal_nan=True)
    out, lse = torch.full_like(qt, 7.0), torch.full((n, hq), 7.0, device="cuda")
    vpb.vp_paged_attention8(dims, qt, _cu([n]), c.kv_len, c.kv, out, lse, ws)
    assert vpb.vp_read_device_error(ws) == 0 and _ran(ws)[0] == kernel
    return _f64(out), _f64(lse)


def _exact(seed, L, d):
    return so.dequantise_rows(*so.quantise_rows(np.random.default_rng(seed).standard_normal((L, 1, d))))


# (tokens, query heads, kernel): items of 8 rows, of 16 rows, tiles
SHAPES = [(1, 2, "rows"), (5, 4, "rows"), (600, 12, "tiles")]


# ------------------------------------------------------------------------------ factors of scores
@pytest.mark.parametrize("n,hq,kernel", SHAPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power,scale", [(-110, 2.0 ** 110), (-125, 1.75 * 2.0 ** 125), (110, 2.0 ** -99), (120, 2.0 ** -119), (120, 0.0),
                                         (-20, 1.1 * 2.0 ** 18)])
def test_scores_whose_factors_are_far_apart(n, hq, kernel, d, power, scale):
    """bf16 rows of q of any size under a scale that brings the scores back to the unit: the weights are those of the
    scores, whatever the products of some of their factors would be."""
    rng = np.random.default_rng(n + d)
    L = 1000
    q = np.zeros((n, hq, d))
    q[..., :4] = rng.integers(-3, 4, (n, hq, 4)) / 4 * 2.0 ** power
    k = np.zeros((L, 1, d))
    k[:, 0, :4] = rng.integers(-7, 8, (L, 4)) / 4
    k[::5] *= 2.0 ** -9                                    # rows of other scales
    scale *= 2.0 ** (2 if power == -20 else 0)
    v = _exact(4, L, d)
    out, lse = _run(q, k, v, BF, scale, kernel, block=0)
    rows = sorted({0, n // 2, n - 1})
    want, want_lse, tol = _tolerance(q[rows], k, v, np.full(len(rows), L), float(np.float32(scale)), BF)
    assert np.all(np.abs(out[rows] - want) <= tol)
    assert np.all(np.abs(lse[rows] - want_lse) <= 4e-5 + 4e-6 * np.abs(want_lse))


@pytest.mark.parametrize("n,hq,kernel", SHAPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,size,scale", [(BF, 2.0 ** 100, 2.0 ** 100), (BF, 2.0 ** 120, 2.0 ** 126), (FP, 1.0, 2.0 ** 126)])
def test_scores_of_zero_under_the_largest_scales(n, hq, kernel, d, dtype, size, scale):
    """q . k = 0 whatever the scale: equal weights."""
    L = 1000
    q, k = np.zeros((n, hq, d)), np.zeros((L, 1, d))
    q[..., 0] = size
    k[:, 0, 1] = 57344.0
    k[::3, 0, 1] = 1.0
    v = _exact(4, L, d)
    out, lse = _run(q, k, v, dtype, scale, kernel, block=0)
    want, _, tol = _tolerance(q[:1], k, v, np.full(1, L), 1.0, dtype)
    assert np.all(np.abs(out - want[:, :1]) <= tol[:, :1]) and np.all(np.abs(lse - math.log(L)) <= 4e-5 + 4e-6 * math.log(L))

"""The 8-bit cache's operators at the ends of their number ranges, against the 64-bit definitions (oracle.streaming):
infinities and NaN in q and under a norm, factors of scores whose products leave 32 bits, channels of one row of q far
apart, values at the smallest and largest scales.

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


# ------------------------------------------------------------------------------ infinities and NaN
@pytest.mark.parametrize("n,hq,kernel", SHAPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_rows_of_q_that_are_not_finite(n, hq, kernel, d, dtype):
    """A row of q with an infinity or a NaN gives NaN; the rows beside it are those of the definition.  (Every key
    with an infinite score of one sign: its softmax has no value either.)"""
    L = 1500
    k, v = _exact(1, L, d), _exact(2, L, d)
    assert (k[:, 0, 3] == 0).sum() < L // 2
    q = _f64(_randn(3, n, hq, d, dtype=dtype))
    bad = np.zeros((n, hq), bool)
    bad[0, 0] = bad[n // 2, hq - 1] = bad[n - 1, hq // 2] = True
    for value in (np.nan, np.inf, -np.inf):
        x = q.copy()
        x[bad, 3] = value
        out, lse = _run(x, k, v, dtype, 0.125, kernel)
        assert np.isnan(out[bad]).all() and not np.isfinite(lse[bad]).any()
        rows = sorted({0, n // 2, n - 1, n // 3})
        want, want_lse, tol = _tolerance(q[rows], k, v, so.row_limits(n, L, 1)[rows], 0.125, dtype)
        good = ~bad[rows]
        assert np.all(np.abs(out[rows] - want)[good] <= tol[good])
        assert np.all(np.abs(lse[rows] - want_lse)[good] <= 4e-5 + 4e-6 * np.abs(want_lse[good]))
        assert np.isfinite(out[~bad]).all() and np.isfinite(lse[~bad]).all()


@pytest.mark.parametrize("n,kernel", [(6, "rows"), (900, "tiles")])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_rows_that_see_nothing_have_zeros_whatever_q_holds(n, kernel, dtype):
    L = 4 if n == 6 else 700
    q = _f64(_randn(3, n, 8, 64, dtype=dtype))
    empty = so.row_limits(n, L, 1) <= 0
    assert empty.sum() == n - L
    q[0], q[1, :, 5] = np.nan, np.inf
    out, lse = _run(q, _exact(1, L, 64), _exact(2, L, 64), dtype, 0.125, kernel)
    assert (out[empty] == 0).all() and np.isneginf(lse[empty]).all() and np.isfinite(out[~empty]).all()


@pytest.mark.parametrize("kind", ["none", "rms", "layer"])
@pytest.mark.parametrize("d,dtype", [(64, BF), (128, FP)])
@pytest.mark.parametrize("T", [1, 7, 3000])
def test_norms_of_rows_that_are_not_finite(kind, d, dtype, T):
    """A head with an infinity or a NaN is NaN after a norm, is marked by its scale in the 8-bit cache with zeros for
    codes, and leaves its neighbours (other heads of the token, other tokens) the bits that they have without it."""
    hq, hkv = 6, 3
    dims = vpb.attn_dims(hq, hkv, d, dtype=dtype)
    x = _randn(4, T, hq + 2 * hkv, d, dtype=dtype)
    gain = 1 + 0.2 * _randn(5, d, dtype=torch.float32)
    hn = vpb.head_norm(kind, 1e-6, q_gain=gain, k_gain=gain) if kind != "none" else None
    rope, pos = vpb.rope_axes(vpb.rope_axes_turns([d // 4, d // 4]).cuda()), torch.arange(2 * T, dtype=torch.int32, device="cuda")
    bad = torch.zeros(T, hq + 2 * hkv, dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[T // 2, hq + 1] = bad[T - 1, hq + hkv + 2] = bad[T // 3, hq - 1] = bad[T // 3, hq + hkv - 1] = True

    def store(t):
        c = Cache8(9, [T], hkv, d, 64)
        q, k = torch.zeros(T, hq, d, dtype=dtype, device="cuda"), torch.zeros(T, hkv, d, dtype=dtype, device="cuda")
        vpb.vp_norm_rope_append(dims, hn, rope, t[:, :hq], t[:, hq:hq + hkv], t[:, hq + hkv:], _cu([T]), c.kv_len,
                                pos, c.kv, q_out=q, k_out=k)
        pg, row = c.at(0, 0, T)
        codes, scales = torch.cat((c.k[pg, :, row], c.v[pg, :, row]), 1), torch.cat((c.ks[pg, :, row], c.vs[pg, :, row]), 1)
        return torch.cat((q, k), 1), codes, scales

    ref = store(x)
    for value in (math.nan, math.inf, -math.inf):
        t = x.clone()
        t[..., 2] = torch.where(bad, torch.full_like(t[..., 2], value), t[..., 2])
        rows, codes, scales = store(t)
        lost, lost8 = bad[:, :hq + hkv], bad[:, hq:]
        assert torch.equal(rows[~lost], ref[0][~lost])
        if kind == "rms" and math.isinf(value):  # what is finite over an infinite root is 0
            pair = torch.arange(d, device="cuda") % (d // 2) == 2
            assert rows[lost][:, pair].isnan().all() and (rows[lost][:, ~pair] == 0).all()
        else:
            hit = ~rows[lost].isfinite()
            assert hit.all() if kind != "none" else hit.any(-1).all()
        assert torch.equal(codes[~lost8], ref[1][~lost8]) and torch.equal(scales[~lost8], ref[2][~lost8])
        assert (codes[lost8] == 0).all() and (scales[lost8] == 255).all()


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d", [64, 128])
def test_norms_of_heads_whose_squares_pass_32_bits(kind, d):
    x = _randn(1, 3, 4, d, dtype=BF)
    x[1, 2] *= 2.0 ** 80
    x[2, :] *= 2.0 ** 50  # squares of 2^100: in range
    gain, bias = (_randn(s, d, dtype=torch.float32) for s in (2, 3))
    out = torch.empty_like(x)
    rope = vpb.rope_axes(torch.zeros(1, 0, dtype=torch.int64, device="cuda"))
    vpb.vp_norm_rope_append(vpb.attn_dims(4, 4, d), vpb.head_norm(kind, 1e-6, k_gain=gain, k_bias=bias), rope, None, x, None,
                            _cu([3]), None, None, None, k_out=out)
    want = so.head_norm(_f64(x), kind, 1e-6, _f64(gain), _f64(bias))
    want[1, 2] = _f64(bias)
    err = 2.0 ** -15 * np.abs(want).max(-1, keepdims=True)  # test_gpu_cache8.py: 32-bit norms
    assert np.all(np.abs(_f64(out) - want) <= err + EPS[BF] * np.abs(want))


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


# ------------------------------------------------------------------------------ channels of q far apart
@pytest.mark.parametrize("n,hq,kernel", SHAPES)
@pytest.mark.parametrize("d", [64, 128])
def test_channels_of_q_far_apart(n, hq, kernel, d):
    """A bf16 row of q keeps its 8 bits down to 2^-31 of its largest magnitude, and below that the multiples of 2^-38
    of the power of two at or below it (halves to even): the weights are those of that row."""
    rng = np.random.default_rng(n)
    L = 1200
    small = rng.integers(128, 256, (n, hq, d)) / 128 * rng.choice([-1, 1], (n, hq, d)) * 2.0 ** rng.integers(-3, 3, (n, hq, d))
    for power in (20, 28, 33, 38, 42, 60):
        q = small.copy()
        q[..., 0] = 1.5 * 2.0 ** power                     # over a channel of k that is 0
        unit = 2.0 ** (power - 38)
        held = np.where(np.abs(q) < 2.0 ** (power - 28), np.round(q / unit) * unit, q)
        assert power > 30 or np.array_equal(held, q)
        k = np.zeros((L, 1, d))
        k[:, 0, 1:9] = rng.integers(-7, 8, (L, 8)) / 4
        v = _exact(6, L, d)
        out, lse = _run(q, k, v, BF, 0.25, kernel, block=0)
        rows = sorted({0, n // 2, n - 1})
        want, want_lse, tol = _tolerance(held[rows], k, v, np.full(len(rows), L), 0.25, BF)
        assert np.all(np.abs(out[rows] - want) <= tol)
        assert np.all(np.abs(lse[rows] - want_lse) <= 4e-5 + 4e-6 * np.abs(want_lse))


# ------------------------------------------------------------------------------ scales of v
@pytest.mark.parametrize("n,hq,kernel", SHAPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,which", [(BF, "smallest"), (BF, "subnormal"), (BF, "largest"), (FP, "smallest"),
                                         (FP, "largest")])
def test_values_at_the_ends_of_the_range(n, hq, kernel, d, dtype, which):
    """Values of one sign under the smallest and the largest scale, with the weight on them and rows of other sizes
    beside them: the output is theirs.  An output of zero, or with a scale a power of two off, would exceed the
    tolerance."""
    rng = np.random.default_rng(d)
    L = 900
    heavy = np.arange(L) % 4 == 1
    q, k = np.zeros((n, hq, d)), np.zeros((L, 1, d))
    q[..., 0] = 1
    k[:, 0, 0] = np.where(heavy, 40.0, 0.0)
    ends = {"smallest": (rng.integers(8, 15, (L, 1, d)) * 2.0 ** rng.integers(0, 6, (L, 1, d)), 2.0 ** -14),
            "subnormal": (rng.integers(1, 8, (L, 1, d)) * 2.0 ** -9, 2.0 ** -14),
            "largest": (rng.integers(8, 15, (L, 1, d)) * 32.0, 2.0 ** 7)}[which]
    v = np.where(heavy[:, None, None], ends[0] * ends[1], so.dequantise_rows(*so.quantise_rows(rng.standard_normal((L, 1, d)))))
    scales = so.quantise_rows(v)[1][heavy]
    assert np.all(scales == (134 if which == "largest" else 113))
    out, _ = _run(q, k, v, dtype, 1.0, kernel, block=0)
    want, _, tol = _tolerance(q[:1], k, v, np.full(1, L), 1.0, dtype)
    assert np.all(want > 0) and np.all(tol < want / 4)
    assert np.all(np.abs(out - want[:, :1]) <= tol[:, :1])


@pytest.mark.parametrize("n,L,hq,kernel", [(1, 30011, 8, "rows"), (3, 12345, 4, "rows"), (200, 9001, 8, "tiles")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_long_contexts_to_the_last_bits_of_the_weights(n, L, hq, kernel, d, dtype):
    """Unit normal q, k and v over many keys (weights from 1 down to 2^-32 of the largest and below)."""
    k, v = _exact(7, L, d), _exact(8, L, d)
    q = _f64(_randn(9, n, hq, d, dtype=dtype))
    out, lse = _run(q, k, v, dtype, 0.35, kernel)
    rows = sorted({0, n // 2, n - 1})
    want, want_lse, tol = _tolerance(q[rows], k, v, so.row_limits(n, L, 1)[rows], 0.35, dtype)
    assert np.all(np.abs(out[rows] - want) <= tol)
    assert np.all(np.abs(lse[rows] - want_lse) <= 4e-5 + 4e-6 * np.abs(want_lse))

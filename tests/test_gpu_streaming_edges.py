"""Streaming attention on the GPU where its kernels' schedules and number ranges end: items cut between
CTAs, large scores, no tokens, against the 64-bit definitions (oracle.streaming)."""
import math

import numpy as np
import pytest
import torch

from oracle import streaming as so
from test_gpu_streaming import BF, FP, Cache, _check_attention, _cu, _dirty_ws, _f64, _randn, vpb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    vpb.lib()


# ------------------------------------------------------------------------------ cut items
@pytest.mark.parametrize("kl,hq,hkv,d,dtype", [
    ([1000], 16, 4, 64, BF),  # four items of 16 tiles: a CTA holds one tile or none
    ([1023, 700, 1500], 4, 2, 64, FP),
    ([777], 8, 1, 128, FP),
    ([640, 5000, 1], 8, 2, 128, BF),
])
def test_cut_items_are_joined_on_every_call(kl, hq, hkv, d, dtype):
    """Single tokens whose items are cut into runs of a few tiles: every call writes every output, the
    same bits each time."""
    B = len(kl)
    dims = vpb.attn_dims(hq, hkv, d, dtype=dtype)
    c = Cache(23, kl, hkv, d, 32, dtype)
    q, cu = _randn(24, B, hq, d, dtype=dtype), _cu([1] * B)
    ws = _dirty_ws(dims, B, B)
    first, first_lse = torch.full_like(q, float("nan")), torch.full((B, hq), float("nan"), device="cuda")
    vpb.vp_paged_attention(dims, q, cu, c.kv_len, c.kv, first, first_lse, ws)
    for b, n in enumerate(kl):
        kd, vd = c.dense[b]
        want = so.seq_attention(_f64(q[b:b + 1]), _f64(kd), _f64(vd), so.row_limits(1, n, 1), 1 / math.sqrt(d))
        _check_attention(_f64(first[b:b + 1]), _f64(first_lse[b:b + 1]), want, dtype, n, float(vd.abs().max()))
    out, lse = torch.empty_like(first), torch.empty_like(first_lse)
    same = torch.ones((), dtype=torch.bool, device="cuda")
    for _ in range(300):
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        vpb.vp_paged_attention(dims, q, cu, c.kv_len, c.kv, out, lse, ws)
        same &= (out == first).all() & (lse == first_lse).all()
    assert same.item()
    assert vpb.vp_read_device_error(ws) == 0


# ------------------------------------------------------------------------------ large scores
def _large_scores(k_rows, q_row, n, d, dtype, scale, sign=1, block=1):
    """A prompt of n tokens whose q and k have a few channels set and the rest zero, checked."""
    dims = vpb.attn_dims(2, 1, d, dtype=dtype, block=block, scale=scale)
    q = torch.zeros(n, 2, d, dtype=dtype, device="cuda")
    k, v = torch.zeros(n, 1, d, dtype=dtype, device="cuda"), _randn(11, n, 1, d, dtype=dtype)
    for ch, x in enumerate(q_row):
        q[..., ch] = sign * x
    for ch, x in enumerate(k_rows):
        k[:, 0, ch] = x.to(dtype).cuda()
    out, lse, ws = torch.full_like(q, float("nan")), torch.empty(n, 2, device="cuda"), _dirty_ws(dims, n, 1)
    vpb.vp_prompt_attention(dims, q, k, v, _cu([n]), out, lse, ws)
    want = so.seq_attention(_f64(q), _f64(k), _f64(v), so.row_limits(n, n, block), float(np.float32(scale)))
    _check_attention(_f64(out), _f64(lse), want, dtype, n, float(v.abs().max()))


@pytest.mark.parametrize("n,d", [(100, 64), (100, 128), (2048, 64), (2048, 128)])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("low", [2 ** 27 + 16, 2 ** 27 + 48, 2 ** 28 - 16])
def test_maximum_that_grows_by_one_unit_in_the_last_place(low, dtype, n, d):
    """log2 scores of `low` in the first half of the keys and low + 16, the next 32-bit value, in the second:
    a threshold of 8 added to the first rounds to the second.  Scale times log2(e) is 1 in 32 bits.

    All products are exact (powers of two times 8 bits) and so are their sums (multiples of 16 below
    2^28); the second half's weights are 2^16 times the first's."""
    scale = 0.6931472
    assert np.float32(scale) * np.float32(1.4426950408889634) == 1
    step = torch.where(torch.arange(n) < n // 2, 0.0, 1.0)
    base = 2 ** 27 if low < 2 ** 28 - 16 else 2 ** 28
    _large_scores([torch.full((n,), base / 16384.0), (low - base) / 16.0 + step], [16384.0, 16.0], n, d, dtype, scale,
                  block=0)


@pytest.mark.parametrize("n,d", [(100, 64), (100, 128), (2048, 64), (2048, 128)])
@pytest.mark.parametrize("dtype,top", [(FP, (59.5, 59.5)), (FP, (30016.0, 20000.0)), (FP, (60000.0, 40000.0)),
                                       (BF, (30080.0, 20096.0)), (BF, (2.2e6, 3.3e6)), (BF, (3.0e9, 2.1e9)),
                                       (BF, (1.1e15, 0.9e15))])
@pytest.mark.parametrize("scale", [1.1, 0.77, 2.9])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_any_size(n, d, dtype, top, scale, sign):
    """Scores up to 10^30, far past where a unit in the last place of one is a whole power of two of its
    weight: equal scores have equal weights and the largest one's is not lost."""
    x = torch.full((n,), top[1])
    x[::3] = top[1] / 2
    _large_scores([x], [top[0]], n, d, dtype, scale, sign)


@pytest.mark.parametrize("n,d", [(100, 64), (2048, 64), (2048, 128)])
@pytest.mark.parametrize("dtype,top", [(FP, (30016.0, 60000.0)), (BF, (3.0e9, 2.1e9))])
@pytest.mark.parametrize("scale", [0.6931472, 0.77, 2.9])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("order", ["rising", "mixed"])
def test_scores_from_small_to_far(n, d, dtype, top, scale, sign, order):
    """Keys whose scores run from 0 to 10^9 and more, small, far and between in one row, in steps that grow
    faster than a unit in the last place of the scores."""
    x = torch.linspace(0, 1, n).to(dtype).float().pow(3) * top[1]
    if order == "mixed":
        x = x[torch.randperm(n, generator=torch.Generator().manual_seed(n))]
    _large_scores([x], [top[0]], n, d, dtype, scale, sign)


# ------------------------------------------------------------------------------ no tokens
def test_calls_without_new_tokens():
    """No new tokens (empty tensors have no address): nothing is done, and nothing refused."""
    c = Cache(3, [70, 5], 2, 64, 16, BF)
    dims = vpb.attn_dims(4, 2, 64)
    q, k = torch.empty(0, 4, 64, dtype=BF, device="cuda"), torch.empty(0, 2, 64, dtype=BF, device="cuda")
    assert q.data_ptr() == 0
    lse = torch.empty(0, 4, device="cuda")
    rope = vpb.rope_options(vpb.rope_turns(64).cuda())
    ws = vpb.attn_workspace(dims, 0, 2)
    k0, v0 = c.k.clone(), c.v.clone()
    for cu, kv_len in ((_cu([0, 0]), c.kv_len), (_cu([]), c.kv_len[:0])):
        vpb.vp_rope_append(dims, rope, q, k, k, cu, kv_len, None, c.kv, q_out=q, k_out=k, ws=ws)
        vpb.vp_prompt_attention(dims, q, k, k, cu, q, lse, ws)
        vpb.vp_paged_attention(dims, q, cu, kv_len, c.kv, q, lse, ws)
    assert vpb.vp_read_device_error(ws) == 0

    def same(a, b):  # NaN in unused slots
        return torch.equal(a.view(torch.int16), b.view(torch.int16))

    assert same(c.k, k0) and same(c.v, v0)


def test_view_stream_example_without_new_tokens():
    import examples.stream_views as ex

    g = torch.Generator(device="cuda").manual_seed(3)
    blocks = [ex.make_block(g, 256, 4, 2)]
    s = ex.ViewStream(blocks, 2, 20, hq=4, hkv=2)
    x = torch.randn(9, 256, generator=g, device="cuda").to(BF)
    assert s.extend(x[:0], [0, 0]).shape == (0, 256) and s.held == [0, 0]
    a = s.extend(x[:6], [4, 2])
    assert s.query(x[:0], [0, 0]).shape == (0, 256) and s.extend(x[:0], [0, 0]).shape == (0, 256)
    assert s.held == [4, 2] and s.errors() == 0
    b = s.extend(x[6:], [3, 0])
    t = ex.ViewStream(blocks, 2, 20, hq=4, hkv=2)
    assert torch.equal(t.extend(x[:6], [4, 2]), a) and torch.equal(t.extend(x[6:], [3, 0]), b)

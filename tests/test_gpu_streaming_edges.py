"""Streaming attention on the GPU where its kernels' schedules and number ranges end: items cut between
CTAs, chains that start anew at mask blocks, large scores, no tokens, against the 64-bit definitions
(oracle.streaming).  Cases that are meant for one of the two kernels check that it ran."""
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


# ------------------------------------------------------------------------------ which kernel
def _ran(ws):
    """(kernel, number of cut items) of the last call that was given `ws`, filled with ones before it.  Each
    CTA leaves 32 bytes in the list behind the error word: a CTA per SM is the tile kernel, more of them
    the kernel for few rows.  An entry's first value is the number of an item's parts."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    recs = ws[256:256 + 32 * 2 * sms].view(torch.int32).view(2 * sms, 8)[:, 0].cpu()
    tiles = bool((recs[sms:] == -1).all())
    assert (recs[:sms] >= 0).all()
    return ("tiles" if tiles else "rows"), int((recs[:sms] > 0).sum())


def _chains_start_anew(group, block):
    """Whether a chain of 128 / group tokens starts at every mask block (at most 1/16 of its rows empty)."""
    n = 128 // group
    return block > n and 16 * (-block % n) <= block


def _lse_and_out(T, hq, d, dtype):
    return (torch.full((T, hq), float("nan"), device="cuda"),
            torch.full((T, hq, d), float("nan"), dtype=dtype, device="cuda"))


# ------------------------------------------------------------------------------ chains at mask blocks
@pytest.mark.parametrize("lens,hq,hkv,d,block,dtype,cut", [
    ([2948], 2, 2, 64, 1374, BF, True),                # two views and part of a third, 11 chains a view
    ([1374, 0, 130, 1, 2748], 4, 1, 64, 1374, FP, True),  # 43 chains a view
    ([2061], 8, 2, 128, 1374, BF, True),
    ([1374, 2061, 77], 3, 3, 128, 1374, FP, True),
    ([1100, 128, 129], 16, 4, 64, 128, BF, True),      # blocks of whole chains
    ([2100, 127, 254], 12, 6, 64, 127, FP, True),
    ([1500, 125], 6, 2, 128, 125, BF, True),           # chains of 42 tokens
    ([777, 250, 251, 749], 16, 16, 128, 250, FP, False),
    ([261, 522, 300], 8, 8, 64, 250, BF, False),
    ([5000], 1, 1, 64, 250, FP, True),
])
def test_prompt_chains_at_mask_blocks(lens, hq, hkv, d, block, dtype, cut):
    assert _chains_start_anew(hq // hkv, block)
    T, B = sum(lens), len(lens)
    dims = vpb.attn_dims(hq, hkv, d, dtype=dtype, block=block)
    qkv = _randn(41, T, hq + 2 * hkv, d, dtype=dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    ws = _dirty_ws(dims, T, B)
    lse, out = _lse_and_out(T, hq, d, dtype)
    vpb.vp_prompt_attention(dims, q, k, v, _cu(lens), out, lse, ws)
    assert vpb.vp_read_device_error(ws) == 0
    kernel, cuts = _ran(ws)
    assert kernel == "tiles" and (cuts > 0) == cut
    t = 0
    for n in lens:
        r = slice(t, t + n)
        if n:
            want = so.seq_attention(_f64(q[r]), _f64(k[r]), _f64(v[r]), so.row_limits(n, n, block), 1 / math.sqrt(d))
            _check_attention(_f64(out[r]), _f64(lse[r]), want, dtype, n, float(v.abs().max()))
        t += n


@pytest.mark.parametrize("ql,kl,hq,hkv,d,page,block,dtype,cut", [
    ([1374], [4122], 4, 4, 64, 64, 1374, BF, True),           # a view over two
    ([1500, 1374], [2874, 4000], 8, 2, 64, 16, 1374, FP, True),   # a chunk that ends inside a view
    ([2748], [2748], 4, 1, 128, 128, 1374, BF, True),
    ([1374, 200], [3000, 9000], 2, 2, 128, 32, 1374, FP, True),
    ([300, 0, 500, 128], [1300, 70, 500, 2000], 8, 2, 64, 64, 128, BF, True),
    ([500, 251], [400, 3000], 4, 4, 128, 16, 250, FP, True),  # more new tokens than the sequence holds
    ([400, 375], [2000, 375], 6, 2, 64, 256, 125, FP, True),
])
def test_paged_chains_at_mask_blocks(ql, kl, hq, hkv, d, page, block, dtype, cut):
    assert _chains_start_anew(hq // hkv, block)
    _paged_case(ql, kl, hq, hkv, d, page, block, dtype, "tiles", cut)


def _paged_case(ql, kl, hq, hkv, d, page, block, dtype, kernel, cut):
    T, B = sum(ql), len(ql)
    dims = vpb.attn_dims(hq, hkv, d, dtype=dtype, block=block)
    c = Cache(42, kl, hkv, d, page, dtype)
    q = _randn(43, T, hq, d, dtype=dtype)
    ws = _dirty_ws(dims, T, B)
    lse, out = _lse_and_out(T, hq, d, dtype)
    vpb.vp_paged_attention(dims, q, _cu(ql), c.kv_len, c.kv, out, lse, ws)
    assert vpb.vp_read_device_error(ws) == 0
    ran, cuts = _ran(ws)
    assert ran == kernel and (cuts > 0) == cut
    t = 0
    for b, (m, n) in enumerate(zip(ql, kl)):
        kd, vd = c.dense[b]
        lim = so.row_limits(m, n, block)
        if m:
            want = so.seq_attention(_f64(q[t:t + m]), _f64(kd), _f64(vd), lim, 1 / math.sqrt(d))
            _check_attention(_f64(out[t:t + m]), _f64(lse[t:t + m]), want, dtype, n, float(vd.abs().max()) if n else 0.0)
            assert (out[t:t + m][torch.from_numpy(lim <= 0).cuda()] == 0).all()
        t += m


# ------------------------------------------------------------------------------ every instance of both kernels
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("ql,kl,block,kernel,cut", [
    ([500], [6001], 1, "tiles", True),
    ([300, 261, 0, 700], [300, 3000, 9, 701], 1, "tiles", True),
    ([600], [4000], 0, "tiles", True),
    ([400, 300], [250, 310], 1, "tiles", False),   # the first has rows that see nothing
    ([1, 1, 1], [3000, 1, 777], 1, "rows", True),
    ([5, 2], [2049, 4000], 1, "rows", True),
    ([3], [9000], 0, "rows", True),
])
def test_paged_instances(ql, kl, block, kernel, cut, d, dtype):
    _paged_case(ql, kl, 8, 2, d, 32, block, dtype, kernel, cut)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lens,hkv,block,kernel,cut", [
    ([3001], 2, 1, "tiles", True),
    ([1800, 33, 900], 2, 0, "tiles", True),
    ([2500], 1, 7, "tiles", True),
    ([3, 400, 3], 1, 1, "rows", True),
])
def test_prompt_instances(lens, hkv, block, kernel, cut, d, dtype):
    T, hq = sum(lens), 4 * hkv
    dims = vpb.attn_dims(hq, hkv, d, dtype=dtype, block=block)
    qkv = _randn(44, T, hq + 2 * hkv, d, dtype=dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    ws = _dirty_ws(dims, T, len(lens))
    lse, out = _lse_and_out(T, hq, d, dtype)
    vpb.vp_prompt_attention(dims, q, k, v, _cu(lens), out, lse, ws)
    assert vpb.vp_read_device_error(ws) == 0
    ran, cuts = _ran(ws)
    assert ran == kernel and (cuts > 0) == cut
    t = 0
    for n in lens:
        r = slice(t, t + n)
        want = so.seq_attention(_f64(q[r]), _f64(k[r]), _f64(v[r]), so.row_limits(n, n, block), 1 / math.sqrt(d))
        _check_attention(_f64(out[r]), _f64(lse[r]), want, dtype, n, float(v.abs().max()))
        t += n


# ------------------------------------------------------------------------------ the place of every value
def _marked_v(n, d, dtype):
    """V [n][1][d] that is 0 but in channel (j / 16) mod d, whose size tells the laps of 16 d keys apart: what
    comes out in a channel is the weight of its keys, so a tile or page taken from elsewhere shows."""
    v = torch.zeros(n, 1, d)
    part = torch.arange(n) // 16
    v[torch.arange(n), 0, part % d] = 200.0 + 24.0 * (part // d % 32).float()
    return v.to(dtype).cuda()  # at most 944: exact in 8 bits (multiples of 8 up to 2^10: bf16 holds multiples of 4)


def _check_marked(got, q, k, v, lim, d, dtype):
    """Tolerances.  Output and weights rounded to the storage type: eps (spread + |out|).  Scores in 32 bits:
    2^-11 spread, as for all inputs of unit normal channels.  fp16 weights are held 2^7 above their value
    relative to a reference at most 2^8 below the row's maximum, so the row's weights sum to 2^7 and more (2^-5
    of that allowed for the reference's own rounding), and one below 2^-14 is off by up to 2^-25:
    n 2^-32 max |v| (1 + 2^-5)."""
    eps = {BF: 2.0 ** -8, FP: 2.0 ** -11}[dtype]
    out, _, spread = so.seq_attention(q, k, v, lim, 1 / math.sqrt(d))
    tol = eps * (spread + np.abs(out)) + 2.0 ** -11 * spread + 2.0 ** -24
    if dtype == FP:
        tol = tol + np.asarray(lim).reshape(-1, 1, 1) * 2.0 ** -32 * 944 * (1 + 2.0 ** -5)
    err = np.abs(got - out)
    assert np.all(err <= tol), f"worst ratio {np.max(err / tol):.3f}"


@pytest.mark.parametrize("n,L,hq,page,kernel", [
    (1, 30011, 8, 1024, "rows"),
    (1, 20000, 16, 16, "rows"),
    (3, 12345, 4, 64, "rows"),
    (300, 9001, 2, 16, "tiles"),
    (200, 30011, 4, 128, "tiles"),
    (129, 70001, 2, 32, "tiles"),
])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [FP, BF])
def test_paged_values_are_those_of_their_keys(n, L, hq, page, kernel, d, dtype):
    dims = vpb.attn_dims(hq, 1, d, dtype=dtype)
    c = Cache(51, [L], 1, d, page, dtype)
    kd, vd = c.dense[0][0], _marked_v(L, d, dtype)
    c.write(0, kd, vd)
    q, ws = _randn(52, n, hq, d, dtype=dtype), _dirty_ws(dims, n, 1)
    out = torch.full_like(q, float("nan"))
    vpb.vp_paged_attention(dims, q, _cu([n]), c.kv_len, c.kv, out, None, ws)
    assert vpb.vp_read_device_error(ws) == 0 and _ran(ws)[0] == kernel
    rows = sorted({0, n // 3, n - 1})  # of a chunk, three tokens
    _check_marked(_f64(out[rows]), _f64(q[rows]), _f64(kd), _f64(vd), so.row_limits(n, L, 1)[rows], d, dtype)


@pytest.mark.parametrize("lens,hq,block,kernel", [([9001], 1, 1, "tiles"), ([700, 5000], 2, 0, "tiles"),
                                                  ([3, 600, 3], 2, 1, "rows")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [FP, BF])
def test_prompt_values_are_those_of_their_keys(lens, hq, block, kernel, d, dtype):
    T = sum(lens)
    dims = vpb.attn_dims(hq, 1, d, dtype=dtype, block=block)
    q, k, v = _randn(53, T, hq, d, dtype=dtype), _randn(54, T, 1, d, dtype=dtype), _marked_v(T, d, dtype)
    ws, out = _dirty_ws(dims, T, len(lens)), torch.full_like(q, float("nan"))
    vpb.vp_prompt_attention(dims, q, k, v, _cu(lens), out, None, ws)
    assert vpb.vp_read_device_error(ws) == 0 and _ran(ws)[0] == kernel
    t = 0
    for n in lens:
        rows = sorted({0, n // 2, n - 1})
        at = [t + r for r in rows]
        _check_marked(_f64(out[at]), _f64(q[at]), _f64(k[t:t + n]), _f64(v[t:t + n]), so.row_limits(n, n, block)[rows],
                      d, dtype)
        t += n


# ------------------------------------------------------------------------------ wide page tables
@pytest.mark.parametrize("ql,kl", [([1] * 20, [13 * i % 300 + 1 for i in range(20)]), ([70, 1, 33], [300, 200, 33]),
                                   ([1] * 63 + [449], [7 * i % 290 + 1 for i in range(63)] + [3000])])
@pytest.mark.parametrize("d,dtype", [(64, BF), (128, FP)])
def test_tables_wider_than_their_sequences(ql, kl, d, dtype):
    """A table for 131,072 tokens a sequence that hold few, its other entries on no page; single tokens and
    a chunk in one call."""
    T, B, hq, hkv, page = sum(ql), len(ql), 8, 2, 64
    dims = vpb.attn_dims(hq, hkv, d, dtype=dtype)
    c = Cache(61, kl, hkv, d, page, dtype)
    table = torch.full((B, 131072 // page), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    kv = vpb.paged_kv(c.k, c.v, table)
    q, ws = _randn(62, T, hq, d, dtype=dtype), _dirty_ws(dims, T, B)
    lse, out = _lse_and_out(T, hq, d, dtype)
    vpb.vp_paged_attention(dims, q, _cu(ql), c.kv_len, kv, out, lse, ws)
    assert vpb.vp_read_device_error(ws) == 0
    t = 0
    for b, (m, n) in enumerate(zip(ql, kl)):
        kd, vd = c.dense[b]
        want = so.seq_attention(_f64(q[t:t + m]), _f64(kd), _f64(vd), so.row_limits(m, n, 1), 1 / math.sqrt(d))
        _check_attention(_f64(out[t:t + m]), _f64(lse[t:t + m]), want, dtype, n, float(vd.abs().max()))
        t += m

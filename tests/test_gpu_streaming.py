"""The streaming operators on the GPU against their 64-bit definitions (oracle.streaming).

Tolerances.  eps: the storage type's unit roundoff, half the distance between neighbours above a
power of two (2^-8 bf16: 8 significant bits; 2^-11 fp16: 11).
rope: products and sums in 32 bits of values of magnitude up to |a| + |b|, angles to 2^-24 turns:
    |err| <= eps |y| + 2^-20 (|a| + |b|); subnormal fp16 results add 2^-25.
attention: the weights are rounded to the storage type (eps each, so eps x spread on the output,
    spread = sum p |v| / sum p), the output once (eps |out|); 32-bit scores of magnitude up to S err by
    d 2^-24 sum |q k| scale, taken as 2^-11 x spread in all for the inputs here (unit normal
    channels); fp16 weights below 2^-14 are subnormal: up to 2^-25 max |v| per key.
log-sum: the scores' error, 2^-22 per exponential, sums of n terms: 4e-5 + 4e-6 |lse|.
"""
import math

import numpy as np
import pytest
import torch

from oracle import streaming as so

pytestmark = pytest.mark.gpu

vpb = pytest.importorskip("paper_2609_23733_gb300.binding")

BF, FP = torch.bfloat16, torch.float16
EPS = {BF: 2.0 ** -8, FP: 2.0 ** -11}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    vpb.lib()


def _f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _cu(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def _randn(seed, *shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _dirty_ws(dims, T, B):
    """A workspace whose contents are arbitrary but for the error word."""
    ws = vpb.attn_workspace(dims, T, B)
    ws[256:].fill_(0xFF)
    return ws


def _check_attention(got, got_lse, want, dtype, n_keys, vmax):
    out, lse, spread = want
    eps = EPS[dtype]
    tol = eps * (spread + np.abs(out)) + 2.0 ** -11 * spread + 2.0 ** -24
    if dtype == FP:
        tol = tol + n_keys * 2.0 ** -25 * vmax
    err = np.abs(got - out)
    assert np.all(np.isfinite(got))
    assert np.all(err <= tol), f"worst excess {np.max(err - tol):.3e}, max err {np.max(err):.3e}"
    if got_lse is not None:
        empty = np.isneginf(lse)
        assert np.array_equal(np.isneginf(got_lse), empty)
        d = np.abs(got_lse[~empty] - lse[~empty])
        assert np.all(d <= 4e-5 + 4e-6 * np.abs(lse[~empty])), f"lse off by {d.max():.3e}"


class Cache:
    """A paged cache with sequences of given lengths in pages in a mixed order; table entries that no
    token uses are -1, and the rest of the pool holds NaN."""

    def __init__(self, seed, kv_lens, hkv, d, page, dtype, extra=2, fill=float("nan")):
        rng = np.random.default_rng(seed)
        self.lens, self.page = list(kv_lens), page
        need = [-(-n // page) for n in kv_lens]
        total = sum(need) + extra
        order = rng.permutation(total)
        table = np.full((len(kv_lens), max(1, max(need, default=1))), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.table_np = table
        self.table = torch.from_numpy(table).cuda()
        self.k = torch.full((total, hkv, page, d), fill, device="cuda", dtype=dtype)
        self.v = torch.full((total, hkv, page, d), fill, device="cuda", dtype=dtype)
        self.kv_len = torch.tensor(kv_lens, dtype=torch.int32, device="cuda")
        self.dense = []
        for b, n in enumerate(kv_lens):
            kd = _randn(1000 * seed + 2 * b, n, hkv, d, dtype=dtype)
            vd = _randn(1000 * seed + 2 * b + 1, n, hkv, d, dtype=dtype)
            self.dense.append((kd, vd))
            self.write(b, kd, vd)
        self.kv = vpb.paged_kv(self.k, self.v, self.table)

    def write(self, b, kd, vd):
        n = kd.shape[0]
        if n == 0:
            return
        j = torch.arange(n, device="cuda")
        pg = self.table[b].long()[j // self.page]
        self.k[pg, :, j % self.page] = kd
        self.v[pg, :, j % self.page] = vd


# ------------------------------------------------------------------------------ rope + append
ROPE_CASES = [
    # (q lens, kv lens, hq, hkv, d, rot, interleaved, page, dtype)
    ([1], [1], 16, 4, 64, 64, False, 64, BF),
    ([1] * 37, list(range(1, 371, 10)), 16, 4, 64, 64, False, 16, BF),
    ([5, 0, 131, 1], [5, 40, 200, 77], 16, 16, 64, 32, True, 32, FP),
    ([300, 17], [1000, 17], 6, 2, 128, 128, False, 128, FP),
    ([261, 3], [261, 2000], 12, 4, 128, 16, True, 1024, BF),
    ([9], [9], 3, 1, 64, 0, False, 16, BF),
    ([2000], [2000], 8, 8, 64, 48, False, 64, BF),
    ([4000, 999], [4000, 1000], 5, 1, 128, 96, True, 64, FP),
]


@pytest.mark.parametrize("ql,kl,hq,hkv,d,rot,inter,page,dtype", ROPE_CASES)
@pytest.mark.parametrize("scale,base_pos", [(1.0, 0), (1.25, 1_000_003)])
def test_rope_append(ql, kl, hq, hkv, d, rot, inter, page, dtype, scale, base_pos):
    T, B = sum(ql), len(ql)
    dims = vpb.attn_dims(hq, hkv, d, dtype=dtype)
    qkv = _randn(5, T, hq + 2 * hkv, d, dtype=dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    c = Cache(3, kl, hkv, d, page, dtype, fill=7.0)
    k0, v0 = c.k.clone(), c.v.clone()
    rope = vpb.rope_options(vpb.rope_turns(rot).cuda(), interleaved=inter, scale=scale)
    pos = None
    pos_np = np.concatenate([np.arange(n - m, n) for m, n in zip(ql, kl)])
    if base_pos:
        pos_np = pos_np + base_pos
        pos = torch.tensor(pos_np, dtype=torch.int32, device="cuda")
    ws = vpb.attn_workspace(dims, T, B)
    q_out, k_out = torch.zeros(T, hq, d, dtype=dtype, device="cuda"), torch.zeros(T, hkv, d, dtype=dtype, device="cuda")
    vpb.vp_rope_append(dims, rope, q, k, v, _cu(ql), c.kv_len, pos, c.kv, q_out=q_out, k_out=k_out, ws=ws)
    torch.cuda.synchronize()
    assert vpb.vp_read_device_error(ws) == 0
    ang = so.rope_angles(pos_np, 10000.0 ** (-2.0 * np.arange(rot // 2) / max(rot, 1)))
    for x, got in ((q, q_out), (k, k_out)):
        x64 = _f64(x)
        want = so.rope(x64, ang, inter, scale)
        mag = scale * np.abs(x64).sum(-1, keepdims=True)  # covers |a| + |b| of every pair
        tol = EPS[dtype] * np.abs(want) + 2.0 ** -20 * np.minimum(mag, 12.0 * scale) + 2.0 ** -25
        assert np.all(np.abs(_f64(got) - want) <= tol)
        assert torch.equal(got[..., rot:], x[..., rot:])  # the rest of the head passes unchanged
    # the cache: the new slots hold exactly k_out and v, everything else is untouched
    t = 0
    for b, (m, n) in enumerate(zip(ql, kl)):
        j = torch.arange(n - m, n, device="cuda")
        pg = c.table[b].long()[j // page]
        k0[pg, :, j % page] = k_out[t:t + m]
        v0[pg, :, j % page] = v[t:t + m]
        t += m
    assert torch.equal(c.k, k0) and torch.equal(c.v, v0)


def test_rope_in_place_and_without_a_cache():
    dims = vpb.attn_dims(8, 2, 64)
    qkv = _randn(9, 500, 12, 64, dtype=BF)
    rope = vpb.rope_options(vpb.rope_turns(64).cuda())
    want_q, want_k = torch.empty(500, 8, 64, dtype=BF, device="cuda"), torch.empty(500, 2, 64, dtype=BF, device="cuda")
    cu = _cu([200, 300])
    vpb.vp_rope_append(dims, rope, qkv[:, :8], qkv[:, 8:10], None, cu, None, None, q_out=want_q, k_out=want_k)
    vpb.vp_rope_append(dims, rope, None, qkv[:, 8:10], None, cu, None, None, k_out=qkv[:, 8:10])
    assert torch.equal(qkv[:, 8:10], want_k)
    vpb.vp_rope_append(dims, rope, qkv[:, :8], want_k.clone(), None, cu, None, None, q_out=qkv[:, :8], k_out=want_k)
    assert torch.equal(qkv[:, :8], want_q)


def test_rope_positions_far_out():
    """Angles stay exact at positions up to 2^31 - 1, where a 32-bit product would be off by turns."""
    pos_np = np.array([0, 1, 2 ** 24 + 1, 2 ** 31 - 1, 123_456_789])
    dims = vpb.attn_dims(1, 1, 64, dtype=FP)
    x = _randn(2, 5, 1, 64, dtype=FP)
    out = torch.empty_like(x)
    rope = vpb.rope_options(vpb.rope_turns(64).cuda())
    vpb.vp_rope_append(dims, rope, None, x, None, _cu([5]), None, torch.tensor(pos_np, dtype=torch.int32, device="cuda"),
                       k_out=out)
    f = 10000.0 ** (-2.0 * np.arange(32) / 64)
    want = so.rope(_f64(x), so.rope_angles(pos_np, f))
    # the table holds 53 significant bits of each frequency: 2^31 x 2^-53 turns at most
    assert np.all(np.abs(_f64(out) - want) <= EPS[FP] * np.abs(want) + 2.0 ** -16)


def test_rope_skips_slots_outside_the_cache():
    """Tokens whose slot is negative, past the table or on a page outside the pool are skipped and
    reported; their neighbours are written."""
    dims = vpb.attn_dims(2, 1, 64)
    table = torch.tensor([[0, 5], [1, 99]], dtype=torch.int32, device="cuda")  # pool of 4 pages: 5, 99 are outside
    kp, vpg = torch.zeros(4, 1, 16, 64, dtype=BF, device="cuda"), torch.zeros(4, 1, 16, 64, dtype=BF, device="cuda")
    kv = vpb.paged_kv(kp, vpg, table)
    x = _randn(1, 24, 4, 64, dtype=BF)
    rope = vpb.rope_options(vpb.rope_turns(64).cuda())
    q_out = torch.empty(24, 2, 64, dtype=BF, device="cuda")
    ws = vpb.attn_workspace(dims, 24, 2)
    kv_len = torch.tensor([18, 10], dtype=torch.int32, device="cuda")  # slots 6 .. 17 and -2 .. 9
    vpb.vp_rope_append(dims, rope, x[:, :2], x[:, 2:3], x[:, 3:], _cu([12, 12]), kv_len, None, kv, q_out=q_out, ws=ws)
    assert vpb.vp_read_device_error(ws) == vpb.VP_DEVERR_PAGE
    assert vpb.vp_read_device_error(ws) == 0
    want = torch.zeros_like(vpg)
    want[0, 0, 6:16] = x[0:10, 3]
    want[1, 0, 0:10] = x[14:24, 3]
    assert torch.equal(vpg, want)
    assert kp[2:].abs().max() == 0


# ------------------------------------------------------------------------------ prompts
PROMPT_CASES = [
    # (lens, hq, hkv, d, block, dtype)
    ([1], 16, 4, 64, 1, BF),
    ([64], 4, 4, 64, 1, FP),
    ([65], 4, 4, 64, 1, BF),
    ([127, 1, 129], 8, 2, 64, 1, BF),
    ([0, 5, 0, 300, 1, 0], 6, 6, 64, 1, FP),
    ([387], 16, 16, 64, 1, BF),
    ([1000, 17, 261], 16, 4, 64, 1, BF),
    ([1000, 17, 261], 16, 4, 64, 261, FP),
    ([700, 64], 4, 2, 64, 0, BF),
    ([523], 3, 1, 64, 7, BF),
    ([300, 41], 5, 1, 64, 1, BF),
    ([90, 33], 128, 1, 64, 1, BF),
    ([65], 2, 2, 128, 1, BF),
    ([513, 255], 4, 4, 128, 1, FP),
    ([900, 1, 77], 12, 4, 128, 1, BF),
    ([770], 14, 2, 128, 64, FP),
    ([258, 259], 8, 2, 128, 0, BF),
    ([2500], 2, 2, 64, 1, BF),
    ([1, 1, 1, 2, 1, 3] * 7, 8, 2, 64, 1, BF),
]


@pytest.mark.parametrize("lens,hq,hkv,d,block,dtype", PROMPT_CASES)
def test_prompt_attention(lens, hq, hkv, d, block, dtype):
    T, B = sum(lens), len(lens)
    dims = vpb.attn_dims(hq, hkv, d, dtype=dtype, block=block)
    qkv = _randn(21, T, hq + 2 * hkv, d, dtype=dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    ws = _dirty_ws(dims, T, B)
    out = torch.full((T, hq, d), float("nan"), dtype=dtype, device="cuda")
    lse = torch.full((T, hq), float("nan"), device="cuda")
    vpb.vp_prompt_attention(dims, q, k, v, _cu(lens), out, lse, ws)
    torch.cuda.synchronize()
    assert vpb.vp_read_device_error(ws) == 0
    t = 0
    for n in lens:
        r = slice(t, t + n)
        want = so.seq_attention(_f64(q[r]), _f64(k[r]), _f64(v[r]), so.row_limits(n, n, block), 1 / math.sqrt(d))
        if n:
            _check_attention(_f64(out[r]), _f64(lse[r]), want, dtype, n, float(v.abs().max()))
        t += n
    again = torch.empty_like(out)
    vpb.vp_prompt_attention(dims, q, k, v, _cu(lens), again, None, ws)
    assert torch.equal(out, again)  # the same bits, with and without the log-sums


def test_prompt_scale_strides_stream_and_tokens_past_the_end():
    """A scale of one's own, an output inside a wider buffer, another stream, tokens past cu[B]."""
    hq, hkv, d, T = 4, 2, 64, 200
    dims = vpb.attn_dims(hq, hkv, d, block=1, scale=-0.31)
    wide = torch.full((T, 3 * hq, d), 5.0, dtype=BF, device="cuda")
    out = wide[:, hq:2 * hq]
    q, k, v = _randn(1, T, hq, d, dtype=BF), _randn(2, T, hkv + 1, d, dtype=BF)[:, :hkv], _randn(3, T, hkv, d, dtype=BF)
    lse = torch.full((T, hq), 9.0, device="cuda")
    ws = _dirty_ws(dims, T, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    vpb.vp_prompt_attention(dims, q, k, v, _cu([100, 70]), out, lse, ws, stream=side)
    side.synchronize()
    for r, n in ((slice(0, 100), 100), (slice(100, 170), 70)):
        want = so.seq_attention(_f64(q[r]), _f64(k[r]), _f64(v[r]), so.row_limits(n, n, 1), -0.31)
        _check_attention(_f64(out[r]), _f64(lse[r]), want, BF, n, 5.0)
    assert (wide[170:] == 5).all() and (wide[:, :hq] == 5).all() and (wide[:, 2 * hq:] == 5).all()
    assert (lse[170:] == 9).all()


@pytest.mark.parametrize("d,bad", [(64, float("nan")), (128, float("inf")), (64, float("-inf"))])
def test_prompt_ignores_what_it_does_not_see(d, bad):
    """Non-finite keys and values of a neighbour sequence, and of later tokens of the same one."""
    dims = vpb.attn_dims(4, 2, d)
    q, k, v = _randn(1, 330, 4, d, dtype=BF), _randn(2, 330, 2, d, dtype=BF), _randn(3, 330, 2, d, dtype=BF)
    cu, ws = _cu([130, 200]), _dirty_ws(dims, 330, 2)
    ref, out = torch.empty_like(q), torch.empty_like(q)
    vpb.vp_prompt_attention(dims, q, k, v, cu, ref, None, ws)
    k2, v2 = k.clone(), v.clone()
    k2[130:], v2[130:] = bad, bad  # the whole second sequence
    vpb.vp_prompt_attention(dims, q, k2, v2, cu, out, None, ws)
    assert torch.equal(out[:130], ref[:130])
    k2, v2 = k.clone(), v.clone()
    k2[250:], v2[250:] = bad, bad  # the second sequence from its token 120 on
    vpb.vp_prompt_attention(dims, q, k2, v2, cu, out, None, ws)
    assert torch.equal(out[:250], ref[:250])
    assert not torch.isfinite(out[250:].float()).any()
    v2 = v.clone()
    v2[250, 1, 3] = bad  # one channel of one value: heads 2 and 3 from token 250 on
    vpb.vp_prompt_attention(dims, q, k, v2, cu, out, None, ws)
    hit = torch.zeros(330, 4, d, dtype=torch.bool, device="cuda")
    hit[250:, 2:, 3] = True
    assert torch.equal(out[~hit], ref[~hit])
    got = out[hit].float()
    assert torch.isnan(got).all() if bad != bad else (got == bad).all()


# ------------------------------------------------------------------------------ paged cache
PAGED_CASES = [
    # (q lens, kv lens, hq, hkv, d, page, block, dtype)
    ([1], [1], 16, 4, 64, 64, 1, BF),
    ([1], [1375], 16, 4, 64, 64, 1, BF),
    ([1], [4097], 4, 4, 128, 16, 1, FP),
    ([1] * 9, [1, 2, 15, 16, 17, 63, 64, 65, 1000], 8, 2, 64, 16, 1, BF),
    ([1, 0, 1, 1], [0, 10, 300, 1], 8, 8, 64, 32, 1, BF),
    ([1, 1], [20000, 33], 16, 2, 128, 128, 1, BF),
    ([1], [30011], 32, 1, 64, 1024, 0, FP),
    ([2, 3, 1], [200, 3, 500], 4, 2, 64, 64, 1, FP),
    ([4, 1], [70, 69], 16, 2, 128, 16, 0, BF),
    ([7], [4], 4, 4, 64, 16, 1, BF),          # more new tokens than the sequence holds: empty rows
    ([100, 3], [64, 0], 4, 2, 64, 16, 1, BF),
    ([261], [783], 16, 4, 64, 64, 261, BF),
    ([130, 1, 64, 17], [1000, 777, 64, 2049], 8, 2, 64, 32, 1, FP),
    ([50, 300], [5000, 300], 6, 2, 128, 16, 7, BF),
    ([33], [9000], 4, 4, 128, 256, 0, FP),
    ([64], [20001], 4, 1, 64, 64, 1, BF),
    ([9], [1], 3, 1, 64, 16, 4, FP),
    ([1] * 70, [13 * i % 611 for i in range(70)], 6, 2, 64, 32, 1, BF),
    ([20], [300], 128, 1, 64, 16, 1, BF),
]


@pytest.mark.parametrize("ql,kl,hq,hkv,d,page,block,dtype", PAGED_CASES)
def test_paged_attention(ql, kl, hq, hkv, d, page, block, dtype):
    T, B = sum(ql), len(ql)
    dims = vpb.attn_dims(hq, hkv, d, dtype=dtype, block=block)
    c = Cache(4, kl, hkv, d, page, dtype)
    q = _randn(77, T, hq, d, dtype=dtype)
    ws = _dirty_ws(dims, T, B)
    out = torch.full((T, hq, d), float("nan"), dtype=dtype, device="cuda")
    lse = torch.full((T, hq), float("nan"), device="cuda")
    vpb.vp_paged_attention(dims, q, _cu(ql), c.kv_len, c.kv, out, lse, ws)
    torch.cuda.synchronize()
    assert vpb.vp_read_device_error(ws) == 0
    t = 0
    for b, (m, n) in enumerate(zip(ql, kl)):
        kd, vd = c.dense[b]
        lim = so.row_limits(m, n, block)
        want = so.seq_attention(_f64(q[t:t + m]), _f64(kd), _f64(vd), lim, 1 / math.sqrt(d))
        if m:
            vmax = float(vd.abs().max()) if n else 0.0
            _check_attention(_f64(out[t:t + m]), _f64(lse[t:t + m]), want, dtype, n, vmax)
            assert (out[t:t + m][torch.from_numpy(lim <= 0).cuda()] == 0).all()
        t += m
    again = torch.empty_like(out)
    vpb.vp_paged_attention(dims, q, _cu(ql), c.kv_len, c.kv, again, None, ws)
    assert torch.equal(out, again)


@pytest.mark.parametrize("n,d", [(1, 64), (5, 64), (3, 128), (90, 64), (90, 128)])
def test_paged_ignores_later_tokens_of_the_chunk(n, d):
    """NaN and infinities in the keys and values of tokens that a row does not see yet."""
    dims = vpb.attn_dims(4, 2, d)
    q = _randn(1, n, 4, d, dtype=BF)
    cu, ws = _cu([n]), _dirty_ws(dims, n, 1)
    ref, out = torch.empty_like(q), torch.empty_like(q)
    c = Cache(8, [500], 2, d, 16, BF)
    vpb.vp_paged_attention(dims, q, cu, c.kv_len, c.kv, ref, None, ws)
    first = n // 2  # the first of the chunk's tokens that goes bad
    kd, vd = (t.clone() for t in c.dense[0])
    kd[500 - n + first:], vd[500 - n + first:] = float("nan"), float("inf")
    c.write(0, kd, vd)
    vpb.vp_paged_attention(dims, q, cu, c.kv_len, c.kv, out, None, ws)
    assert torch.equal(out[:first], ref[:first])
    assert not torch.isfinite(out[first:].float()).any()
    kd, vd = (t.clone() for t in c.dense[0])
    vd[500 - n + first, 0, 1] = float("-inf")  # one channel: heads 0 and 1 from that token on
    c.write(0, kd, vd)
    vpb.vp_paged_attention(dims, q, cu, c.kv_len, c.kv, out, None, ws)
    hit = torch.zeros(n, 4, d, dtype=torch.bool, device="cuda")
    hit[first:, :2, 1] = True
    assert torch.equal(out[~hit], ref[~hit]) and (out[hit] == float("-inf")).all()


@pytest.mark.parametrize("ql", [[1, 1, 1], [60, 1, 200]])
def test_paged_reports_lengths_and_pages_outside_the_cache(ql):
    """A length past the table is clamped and reported, a page id outside the pool is reported; the
    other sequences keep their results."""
    dims = vpb.attn_dims(4, 2, 64)
    T = sum(ql)
    c = Cache(2, [300, 333, 400], 2, 64, 16, BF)
    q = _randn(1, T, 4, 64, dtype=BF)
    ws = _dirty_ws(dims, T, 3)
    ref, out = torch.empty_like(q), torch.empty_like(q)
    vpb.vp_paged_attention(dims, q, _cu(ql), c.kv_len, c.kv, ref, None, ws)
    assert vpb.vp_read_device_error(ws) == 0
    c.kv_len[2] = 10 ** 9  # the table is 25 pages wide: clamped to the 400 tokens it holds
    c.table[1, 3] = 1 << 20
    vpb.vp_paged_attention(dims, q, _cu(ql), c.kv_len, c.kv, out, None, ws)
    assert vpb.vp_read_device_error(ws) == vpb.VP_DEVERR_PAGE
    assert torch.equal(out[:ql[0]], ref[:ql[0]]) and torch.equal(out[ql[0] + ql[1]:], ref[ql[0] + ql[1]:])
    c.kv_len[2] = -5  # a negative length is an empty sequence
    vpb.vp_paged_attention(dims, q, _cu(ql), c.kv_len, c.kv, out, None, ws)
    assert vpb.vp_read_device_error(ws) == vpb.VP_DEVERR_PAGE
    assert (out[ql[0] + ql[1]:] == 0).all()


@pytest.mark.parametrize("n", [1, 100])
def test_paged_pool_past_32_bit_offsets(n):
    """Pages whose elements lie past 2^31, and whose bytes lie past 2^32, in a large pool."""
    hkv, d, page, L = 4, 64, 64, 300
    pages = (2 ** 31 + 2 ** 28) // (hkv * page * d)
    k = torch.empty(pages, hkv, page, d, dtype=BF, device="cuda")
    v = torch.empty(pages, hkv, page, d, dtype=BF, device="cuda")
    ids = torch.tensor([[pages - 1, 0, pages - 7, pages // 2, pages - 2]], dtype=torch.int32, device="cuda")
    kd, vd = _randn(1, L, hkv, d, dtype=BF), _randn(2, L, hkv, d, dtype=BF)
    kv_len = torch.tensor([L], dtype=torch.int32, device="cuda")
    kv = vpb.paged_kv(k, v, ids)
    dims = vpb.attn_dims(8, hkv, d)
    none = vpb.rope_options(torch.empty(0, dtype=torch.int64, device="cuda"))
    vpb.vp_rope_append(dims, none, None, kd, vd, _cu([L]), kv_len, None, kv)  # written by the append
    q = _randn(3, n, 8, d, dtype=BF)
    out, lse, ws = torch.empty_like(q), torch.empty(n, 8, device="cuda"), _dirty_ws(dims, n, 1)
    vpb.vp_paged_attention(dims, q, _cu([n]), kv_len, kv, out, lse, ws)
    assert vpb.vp_read_device_error(ws) == 0
    want = so.seq_attention(_f64(q), _f64(kd), _f64(vd), so.row_limits(n, L, 1), 0.125)
    _check_attention(_f64(out), _f64(lse), want, BF, L, 6.0)


def test_growing_scores_and_far_maxima():
    """Scores that rise along the keys (the running maximum moves at every tile), and one key far
    above all others."""
    dims = vpb.attn_dims(2, 1, 64, dtype=FP, scale=1.0)
    for n in (1, 40):
        q = torch.zeros(n, 2, 64, dtype=FP, device="cuda")
        q[..., 0] = 1
        kd, vd = torch.zeros(2000, 1, 64, dtype=FP, device="cuda"), _randn(4, 2000, 1, 64, dtype=FP)
        kd[:, 0, 0] = torch.arange(2000, device="cuda") * 0.05
        for case in range(2):
            if case == 1:
                kd[:, 0, 0] = 0
                kd[700, 0, 0] = 200
            c = Cache(6, [2000], 1, 64, 32, FP)
            c.write(0, kd, vd)
            out, lse, ws = torch.empty_like(q), torch.empty(n, 2, device="cuda"), _dirty_ws(dims, n, 1)
            vpb.vp_paged_attention(dims, q, _cu([n]), c.kv_len, c.kv, out, lse, ws)
            want = so.seq_attention(_f64(q), _f64(kd), _f64(vd), so.row_limits(n, 2000, 1), 1.0)
            _check_attention(_f64(out), _f64(lse), want, FP, 2000, 6.0)


@pytest.mark.parametrize("n,d", [(100, 64), (100, 128), (2048, 64), (2048, 128)])
@pytest.mark.parametrize("at", [0, 0.5, 1])
def test_light_keys_beside_a_heavy_one(n, d, at):
    """One key whose weight is 2^23.4 times that of each other one, with V zero there: what comes out is
    the light keys' sum.  Tolerance, relative: fp16 keeps a weight, raised by 2^7, to 2^-25, so
    2^-25 / 2^(7 - 23.4); the output's rounding; scores to 2^-16."""
    scale = 16.2
    dims = vpb.attn_dims(2, 1, d, dtype=FP, block=0, scale=scale)
    q = torch.zeros(n, 2, d, dtype=FP, device="cuda")
    k, v = torch.zeros(n, 1, d, dtype=FP, device="cuda"), torch.full((n, 1, d), 1000.0, dtype=FP, device="cuda")
    heavy = int(at * (n - 1))
    q[..., 0] = 1
    k[heavy, 0, 0] = 1
    v[heavy] = 0
    out, lse, ws = torch.empty_like(q), torch.empty(n, 2, device="cuda"), _dirty_ws(dims, n, 1)
    vpb.vp_prompt_attention(dims, q, k, v, _cu([n]), out, lse, ws)
    want, want_lse, _ = so.seq_attention(_f64(q), _f64(k), _f64(v), so.row_limits(n, n, 0), scale)
    tol = 2.0 ** (scale * math.log2(math.e) - 32) + 2.0 ** -11 + 2.0 ** -16
    assert np.all(np.abs(_f64(out) - want) <= tol * want)
    assert np.all(np.abs(_f64(lse) - want_lse) <= 4e-5 + 4e-6 * np.abs(want_lse))


@pytest.mark.parametrize("n,d", [(100, 64), (100, 128), (2048, 64), (2048, 128)])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_past_the_precision_of_32_bits(n, d, dtype, sign):
    """Scores of 1.1 2^25 and 1.1 2^24: a unit in the last place of the maximum is 4 and more."""
    dims = vpb.attn_dims(2, 1, d, dtype=dtype, block=1, scale=1.1)
    q = torch.zeros(n, 2, d, dtype=dtype, device="cuda")
    k, v = torch.zeros(n, 1, d, dtype=dtype, device="cuda"), _randn(11, n, 1, d, dtype=dtype)
    q[..., 0] = sign * 4096
    k[:, 0, 0] = 8192
    k[::3, 0, 0] = 4096
    out, lse, ws = torch.empty_like(q), torch.empty(n, 2, device="cuda"), _dirty_ws(dims, n, 1)
    vpb.vp_prompt_attention(dims, q, k, v, _cu([n]), out, lse, ws)
    want = so.seq_attention(_f64(q), _f64(k), _f64(v), so.row_limits(n, n, 1), 1.1)
    _check_attention(_f64(out), _f64(lse), want, dtype, n, float(v.abs().max()))


def test_chunks_through_the_cache_equal_the_whole_prompt():
    """A prompt attended at once, and the same tokens appended and attended in chunks and single
    tokens: the rotated q and k are the same bits, the outputs agree within both sides' rounding."""
    hq, hkv, d, L = 8, 2, 64, 420
    dims = vpb.attn_dims(hq, hkv, d)
    qkv = _randn(31, L, hq + 2 * hkv, d, dtype=BF)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    rope = vpb.rope_options(vpb.rope_turns(64).cuda())
    qr, kr = torch.empty(L, hq, d, dtype=BF, device="cuda"), torch.empty(L, hkv, d, dtype=BF, device="cuda")
    vpb.vp_rope_append(dims, rope, q, k, None, _cu([L]), None, None, q_out=qr, k_out=kr)
    whole, ws = torch.empty_like(qr), _dirty_ws(dims, L, 1)
    vpb.vp_prompt_attention(dims, qr, kr, v, _cu([L]), whole, None, ws)
    c = Cache(1, [L], hkv, d, 16, BF)
    c.k.fill_(float("nan"))
    c.v.fill_(float("nan"))
    at = 0
    parts = []
    for n in (200, 1, 1, 37, 1, 130, 50):
        r = slice(at, at + n)
        at += n
        kv_len = torch.tensor([at], dtype=torch.int32, device="cuda")
        qc, oc = torch.empty(n, hq, d, dtype=BF, device="cuda"), torch.empty(n, hq, d, dtype=BF, device="cuda")
        vpb.vp_rope_append(dims, rope, q[r], k[r], v[r], _cu([n]), kv_len, None, c.kv, q_out=qc)
        assert torch.equal(qc, qr[r])
        vpb.vp_paged_attention(dims, qc, _cu([n]), kv_len, c.kv, oc, None, ws)
        parts.append(oc)
    want = so.seq_attention(_f64(qr), _f64(kr), _f64(v), so.row_limits(L, L, 1), 0.125)
    _check_attention(_f64(torch.cat(parts)), None, want, BF, L, 6.0)
    _check_attention(_f64(whole), None, want, BF, L, 6.0)


# ------------------------------------------------------------------------------ together
def test_view_stream_example():
    """The example's stack: views streamed through the cache against all views attended at once, and the
    block's tokens against the 64-bit block."""
    import examples.stream_views as ex

    P, D, views = 70, 256, 5
    g = torch.Generator(device="cuda").manual_seed(3)
    blocks = [ex.make_block(g, D, 4, 2) for _ in range(2)]
    x = torch.randn(views * P, D, generator=g, device="cuda").to(BF)
    kw = dict(hq=4, hkv=2, block_tokens=P)
    whole = ex.ViewStream(blocks, 1, views * P, **kw)
    want = whole.extend(x, [views * P])
    stream = ex.ViewStream(blocks, 2, views * P + 3, page_size=16, **kw)
    got = [stream.extend(torch.cat((x[:2 * P], x[:P])), [2 * P, P])[:2 * P]]  # a second sequence beside it
    got.append(stream.extend(x[2 * P:3 * P], [P, 0]))
    got.append(stream.extend(torch.cat((x[3 * P:], x[P:2 * P])), [2 * P, P])[:2 * P])
    got = torch.cat(got)
    assert whole.errors() == 0 and stream.errors() == 0 and stream.held == [5 * P, 2 * P]
    # Both sides round at the same points; where sums fall in another order a rounding may flip, and
    # flips propagate through two blocks: a few bf16 steps of the residual stream at most.
    d = (got.float() - want.float()).abs()
    assert d.max() <= 4 * 2.0 ** -7 * want.float().abs().max() and d.mean() <= 2.0 ** -9 * want.float().abs().mean()
    # a query is not kept
    q = stream.query(x[:3], [2, 1])
    assert q.shape == (3, D) and stream.held == [5 * P, 2 * P]
    with pytest.raises(ValueError):
        stream.extend(x[:4], [4, 0])
    # one block in 64 bits
    one = ex.ViewStream(blocks[:1], 1, views * P, **kw)
    y = _f64(one.extend(x, [views * P]))
    w = {k: _f64(v) for k, v in blocks[0].items()}
    X = _f64(x)

    def ln(t, gm, bt):
        m, s = t.mean(-1, keepdims=True), t.var(-1, keepdims=True)
        return (t - m) / np.sqrt(s + 1e-6) * gm + bt

    qkv = (ln(X, w["ln1_g"], w["ln1_b"]) @ w["w_qkv"].T + w["b_qkv"]).reshape(-1, 8, 64)
    ang = so.rope_angles(np.arange(views * P), 10000.0 ** (-2.0 * np.arange(32) / 64))
    o = so.seq_attention(so.rope(qkv[:, :4], ang), so.rope(qkv[:, 4:6], ang), qkv[:, 6:],
                         so.row_limits(views * P, views * P, P), 0.125)[0]
    X = X + w["ls1"] * (o.reshape(-1, 256) @ w["w_o"].T + w["b_o"])
    h = ln(X, w["ln2_g"], w["ln2_b"]) @ w["w_fc1"].T + w["b_fc1"]
    h = 0.5 * h * (1 + np.vectorize(math.erf)(h / math.sqrt(2)))
    X = X + w["ls2"] * (h @ w["w_fc2"].T + w["b_fc2"])
    err = np.abs(y - X)
    # about ten bf16 roundings on the way (QKV, rotation, P, Y, LN2, hidden, two residual sums)
    assert err.max() <= 10 * 2.0 ** -8 * np.abs(X).max() and err.mean() <= 2.0 ** -7 * np.abs(X).mean()


def test_calls_in_a_graph_follow_their_inputs():
    """A captured step replayed after its inputs changed (lengths, tokens, pages) computes on the new ones."""
    dims = vpb.attn_dims(8, 2, 64)
    c = Cache(11, [700, 90], 2, 64, 32, BF)
    k = _randn(5, 2, 2, 64, dtype=BF)
    q, out = _randn(6, 2, 8, 64, dtype=BF), torch.empty(2, 8, 64, dtype=BF, device="cuda")
    qr = torch.empty_like(q)
    cu, ws = _cu([1, 1]), _dirty_ws(dims, 2, 2)
    rope = vpb.rope_options(vpb.rope_turns(64).cuda())
    kv_len = c.kv_len.clone()

    def step():
        vpb.vp_rope_append(dims, rope, q, k, k, cu, kv_len, None, c.kv, q_out=qr)
        vpb.vp_paged_attention(dims, qr, cu, kv_len, c.kv, out, None, ws)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([700, 90], [650, 33], [1, 64]):
        kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        q.copy_(_randn(60 + lens[0], 2, 8, 64, dtype=BF))
        graph.replay()
        got = out.clone()
        out.zero_()
        step()
        assert torch.equal(got, out)


@pytest.mark.parametrize("n,page", [(1, 16), (40, 64)])
def test_many_sequences(n, page):
    """More sequences than a CTA has threads (the scans of the lengths go in rounds), some of them empty."""
    B, hq, hkv, d = 700, 4, 1, 64
    rng = np.random.default_rng(n)
    ql = [int(x) for x in rng.integers(0, n + 1, B)]
    kl = [int(m + x) if i % 5 else m for i, (m, x) in enumerate(zip(ql, rng.integers(0, 200, B)))]
    dims = vpb.attn_dims(hq, hkv, d)
    T = sum(ql)
    c = Cache(12, kl, hkv, d, page, BF)
    q = _randn(5, T, hq, d, dtype=BF)
    ws = _dirty_ws(dims, T, B)
    out, lse = torch.full_like(q, float("nan")), torch.full((T, hq), float("nan"), device="cuda")
    vpb.vp_paged_attention(dims, q, _cu(ql), c.kv_len, c.kv, out, lse, ws)
    assert vpb.vp_read_device_error(ws) == 0
    qd, od, ld = _f64(q), _f64(out), _f64(lse)
    t = 0
    for b, (m, length) in enumerate(zip(ql, kl)):
        if m:
            kd, vd = c.dense[b]
            want = so.seq_attention(qd[t:t + m], _f64(kd), _f64(vd), so.row_limits(m, length, 1), 0.125)
            _check_attention(od[t:t + m], ld[t:t + m], want, BF, length, 6.0)
        t += m
    # prompts: the same query rows over themselves
    k = _randn(6, T, hkv, d, dtype=BF)
    vpb.vp_prompt_attention(dims, q, k, k, _cu(ql), out, lse, ws)
    assert vpb.vp_read_device_error(ws) == 0
    kd, od, ld = _f64(k), _f64(out), _f64(lse)
    t = 0
    for m in ql:
        if m:
            r = slice(t, t + m)
            _check_attention(od[r], ld[r], so.seq_attention(qd[r], kd[r], kd[r], so.row_limits(m, m, 1), 0.125), BF, m, 6.0)
        t += m


@pytest.mark.parametrize("d,dtype", [(64, BF), (128, FP)])
@pytest.mark.parametrize("B,most,hkv", [(50, 511, 12), (3, 256, 2), (90, 130, 3)])
def test_short_contexts(B, most, hkv, d, dtype):
    """Caches of few pages, more and fewer items than CTAs, chunks of 0 to 3 tokens."""
    rng = np.random.default_rng(most)
    ql = [int(x) for x in rng.integers(0, 4, B)]
    kl = [max(m, int(x)) for m, x in zip(ql, rng.integers(0, most + 1, B))]
    kl[B // 2] = most
    hq = 2 * hkv
    dims = vpb.attn_dims(hq, hkv, d, dtype=dtype)
    T = sum(ql)
    c = Cache(17, kl, hkv, d, 32, dtype)
    q = _randn(18, T, hq, d, dtype=dtype)
    ws = _dirty_ws(dims, T, B)
    out, lse = torch.full_like(q, float("nan")), torch.full((T, hq), float("nan"), device="cuda")
    vpb.vp_paged_attention(dims, q, _cu(ql), c.kv_len, c.kv, out, lse, ws)
    assert vpb.vp_read_device_error(ws) == 0
    qd, od, ld = _f64(q), _f64(out), _f64(lse)
    t = 0
    for b, (m, length) in enumerate(zip(ql, kl)):
        if m:
            kd, vd = c.dense[b]
            want = so.seq_attention(qd[t:t + m], _f64(kd), _f64(vd), so.row_limits(m, length, 1), 1 / math.sqrt(d))
            _check_attention(od[t:t + m], ld[t:t + m], want, dtype, length, float(vd.abs().max()) if length else 0.0)
        t += m

"""Streaming attention on the GPU where its kernels' schedules and number ranges end: items cut between
CTAs, against the 64-bit definitions (oracle.streaming)."""
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

"""Attention over packed and 16-bit paged keys where q is large and the scale small, against the 64-bit definition
(oracle.streaming).  Tolerances: bf16 weights are off by 2^-8 of themselves, scores in 32 bits by 2^-11, the output by its
own rounding; log-sums as in test_gpu_streaming.py."""
import numpy as np
import pytest
import torch

from oracle import streaming as so

pytestmark = pytest.mark.gpu

vpb = pytest.importorskip("paper_2609_23733_gb300.binding")

BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    vpb.lib()


def _bf(x):
    return torch.from_numpy(x).to(BF).cuda()


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("n,hq", [(1, 2), (5, 4), (900, 12)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power,scale", [(120, 2.0 ** -119), (105, 1.3 * 2.0 ** -104), (120, 2.0 ** -145), (120, 0.0), (90, 0.0)])
def test_large_q_under_small_scales(paged, n, hq, d, power, scale):
    rng = np.random.default_rng(n + d)
    L = 1000 if paged else n
    q, k = np.zeros((n, hq, d)), np.zeros((L, 1, d))
    q[..., :4] = rng.integers(-3, 4, (n, hq, 4)) / 4 * 2.0 ** power
    k[:, 0, :4] = rng.integers(-7, 8, (L, 4)) / 4
    vt = _bf(rng.standard_normal((L, 1, d)))
    v = vt.double().cpu().numpy()
    dims = vpb.attn_dims(hq, 1, d, dtype=BF, block=0, scale=scale)
    qt, kt, cu = _bf(q), _bf(k), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    assert np.array_equal(qt.double().cpu().numpy(), q)
    out, lse, ws = torch.empty_like(qt), torch.empty(n, hq, device="cuda"), vpb.attn_workspace(dims, n, 1)
    if paged:
        pad = torch.zeros(1024 - L, 1, d, dtype=BF, device="cuda")
        pool = [torch.cat((t, pad)).view(16, 64, 1, d).transpose(1, 2).contiguous() for t in (kt, vt)]
        kv = vpb.paged_kv(*pool, torch.arange(16, dtype=torch.int32, device="cuda")[None])
        vpb.vp_paged_attention(dims, qt, cu, torch.tensor([L], dtype=torch.int32, device="cuda"), kv, out, lse, ws)
    else:
        vpb.vp_prompt_attention(dims, qt, kt, vt, cu, out, lse, ws)
    assert vpb.vp_read_device_error(ws) == 0
    rows = sorted({0, n // 2, n - 1})
    want, want_lse, spread = so.seq_attention(q[rows], k, v, np.full(len(rows), L), float(np.float32(scale)))
    got, got_lse = out.double().cpu().numpy()[rows], lse.double().cpu().numpy()[rows]
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * (np.abs(want) + spread) + 2.0 ** -11 * spread)
    assert np.all(np.abs(got_lse - want_lse) <= 4e-5 + 4e-6 * np.abs(want_lse))

"""The streaming operators without a GPU: argument checks of the C entry points (before any device is
touched), of the binding, and the rotary tables."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2609_23733_gb300 import binding as vpb
from paper_2609_23733_gb300 import build

OK, INVALID, SHAPE, ALIGN, WORKSPACE, DEVICE = 0, 1, 2, 3, 6, 7
A = 0x10000  # an aligned address that is never read
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(build.LIB):
        build.build()
    return vpb.lib()


def _dims(hq=16, hkv=4, d=64, dtype=0, block=1, scale=0.125):
    return vpb.VpAttnDims(hq, hkv, d, dtype, block, scale)


def _kv(k=A, v=A, table=A, n=8, ps=64, width=4):
    return vpb.VpPagedKv(k, v, table, n, ps, width)


def _rope(turns=A, rot=64, inter=0, scale=1.0):
    return vpb.VpRopeOptions(turns, rot, inter, scale)


def _prompt(lib, dm, T=10, B=2, q=A, qs=1024, k=A, ks=256, v=A, vs=256, cu=A, out=A, os_=1024, lse=A, ws=A, n=BIG):
    return lib.vp_prompt_attention(None if dm is None else ctypes.byref(dm), T, B, q, qs, k, ks, v, vs, cu, out, os_,
                                   lse, ws, n, None)


def _paged(lib, dm, T=10, B=2, q=A, qs=1024, cu=A, lens=A, kv=None, out=A, os_=1024, lse=A, ws=A, n=BIG, no_kv=False):
    kv = _kv() if kv is None else kv
    return lib.vp_paged_attention(ctypes.byref(dm), T, B, q, qs, cu, lens, None if no_kv else ctypes.byref(kv), out,
                                  os_, lse, ws, n, None)


def _append(lib, dm, rope=None, T=10, B=2, q=A, qs=1024, k=A, ks=256, v=A, vs=256, cu=A, lens=A, pos=None, kv=None,
            qo=A, qos=1024, ko=None, kos=0, ws=None, n=0, no_kv=False, no_rope=False):
    kv = _kv() if kv is None else kv
    rope = _rope() if rope is None else rope
    return lib.vp_rope_append(ctypes.byref(dm), None if no_rope else ctypes.byref(rope), T, B, q, qs, k, ks, v, vs, cu,
                              lens, pos, None if no_kv else ctypes.byref(kv), qo, qos, ko, kos, ws, n, None)


# Without a device a call that passes every check reports that (nothing is enqueued either way).
def _passes(status):
    return status == (DEVICE if not torch.cuda.is_available() else OK)


pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses here are not real")


@pytest.mark.parametrize("dm,want", [
    (_dims(), None), (_dims(d=128, dtype=1), None), (_dims(hq=128, hkv=1), None), (_dims(hq=6, hkv=2), None),
    (_dims(block=0), None), (_dims(block=1374), None), (_dims(scale=-1.0), None), (_dims(scale=0.0), None),
    (_dims(d=32), SHAPE), (_dims(d=96), SHAPE), (_dims(hq=0, hkv=0), SHAPE), (_dims(hq=16, hkv=5), SHAPE),
    (_dims(hq=2, hkv=4), SHAPE), (_dims(hq=129, hkv=1), SHAPE), (_dims(hq=16, hkv=-4), SHAPE),
    (_dims(dtype=2), INVALID), (_dims(dtype=-1), INVALID), (_dims(block=-1), INVALID),
    (_dims(scale=float("nan")), INVALID), (_dims(scale=float("inf")), INVALID)])
def test_dims(lib, dm, want):
    n = ctypes.c_size_t(0)
    st = lib.vp_attn_workspace_size(ctypes.byref(dm), 10, 2, ctypes.byref(n))
    assert st == (OK if want is None else want)
    wide = dict(qs=1 << 14, os_=1 << 14)
    st = _prompt(lib, dm, ks=1 << 14, vs=1 << 14, **wide)
    assert _passes(st) if want is None else st == want
    st = _paged(lib, dm, **wide)
    assert _passes(st) if want is None else st == want
    st = _append(lib, dm, qs=1 << 14, ks=1 << 14, vs=1 << 14, qos=1 << 14)
    assert _passes(st) if want is None else st == want


def test_workspace_size(lib):
    dm, n = _dims(), ctypes.c_size_t(0)
    assert lib.vp_attn_workspace_size(None, 10, 2, ctypes.byref(n)) == INVALID
    assert lib.vp_attn_workspace_size(ctypes.byref(dm), 10, 2, None) == INVALID
    assert lib.vp_attn_workspace_size(ctypes.byref(dm), -1, 2, ctypes.byref(n)) == INVALID
    assert lib.vp_attn_workspace_size(ctypes.byref(dm), 10, 0, ctypes.byref(n)) == SHAPE
    assert lib.vp_attn_workspace_size(ctypes.byref(dm), 0, 0, ctypes.byref(n)) == OK
    assert lib.vp_attn_workspace_size(ctypes.byref(dm), (1 << 30) + 1, 2, ctypes.byref(n)) == SHAPE
    small = vpb.vp_attn_workspace_size(vpb.attn_dims(16, 4, 64), 64, 64)
    assert 0 < small <= vpb.vp_attn_workspace_size(vpb.attn_dims(16, 4, 64), 1 << 17, 64) < 1 << 28
    assert _prompt(lib, dm, n=small - 1) == WORKSPACE and _paged(lib, dm, n=small - 1) == WORKSPACE
    assert _prompt(lib, dm, ws=None) == WORKSPACE and _paged(lib, dm, ws=None) == WORKSPACE
    assert _prompt(lib, dm, ws=A + 8) == ALIGN and _paged(lib, dm, ws=A + 8) == ALIGN
    assert _append(lib, dm, ws=A, n=255) == WORKSPACE


def test_counts(lib):
    dm = _dims()
    for call in (_prompt, _paged, _append):
        assert call(lib, dm, T=0) == OK and call(lib, dm, T=0, B=0) == OK  # nothing to do
        assert call(lib, dm, T=-1) == INVALID and call(lib, dm, B=-1) == INVALID
        assert call(lib, dm, T=5, B=0) == SHAPE
        assert call(lib, dm, cu=None) == INVALID
        assert _passes(call(lib, dm))


@pytest.mark.parametrize("name,stride,heads", [("q", "qs", 16), ("k", "ks", 4), ("v", "vs", 4), ("out", "os_", 16)])
def test_prompt_tensors(lib, name, stride, heads):
    dm = _dims()
    assert _prompt(lib, dm, **{name: None}) == INVALID
    assert _prompt(lib, dm, **{name: A + 2}) == ALIGN
    assert _prompt(lib, dm, **{stride: heads * 64 - 8}) == SHAPE
    assert _prompt(lib, dm, **{stride: heads * 64 + 4}) == ALIGN
    assert _prompt(lib, dm, **{stride: -1024}) == SHAPE
    assert _passes(_prompt(lib, dm, **{stride: 1 << 20}))
    assert _passes(_prompt(lib, dm, lse=None))


def test_paged_tensors_and_cache(lib):
    dm = _dims()
    for name, stride in (("q", "qs"), ("out", "os_")):
        assert _paged(lib, dm, **{name: None}) == INVALID
        assert _paged(lib, dm, **{name: A + 2}) == ALIGN
        assert _paged(lib, dm, **{stride: 1016}) == SHAPE
    assert _paged(lib, dm, lens=None) == INVALID
    assert _paged(lib, dm, no_kv=True) == INVALID
    for bad in (_kv(k=None), _kv(v=None), _kv(table=None)):
        assert _paged(lib, dm, kv=bad) == INVALID and _append(lib, dm, kv=bad) == INVALID
    for bad in (_kv(k=A + 8), _kv(v=A + 8)):
        assert _paged(lib, dm, kv=bad) == ALIGN and _append(lib, dm, kv=bad) == ALIGN
    for bad in (_kv(ps=8), _kv(ps=24), _kv(ps=2048), _kv(ps=0), _kv(ps=-64), _kv(n=0), _kv(width=0)):
        assert _paged(lib, dm, kv=bad) == SHAPE and _append(lib, dm, kv=bad) == SHAPE
    for ps in (16, 32, 64, 128, 256, 512, 1024):
        assert _passes(_paged(lib, dm, kv=_kv(ps=ps)))


def test_append_tensors_and_rotation(lib):
    dm = _dims()
    assert _append(lib, dm, no_rope=True) == INVALID
    for rot in (8, 24, 80, 128, -16):
        assert _append(lib, dm, rope=_rope(rot=rot)) == SHAPE
    for rot in (0, 16, 48, 64):
        assert _passes(_append(lib, dm, rope=_rope(rot=rot)))
    assert _append(lib, dm, rope=_rope(turns=None)) == INVALID
    assert _passes(_append(lib, dm, rope=_rope(turns=None, rot=0)))
    assert _append(lib, dm, rope=_rope(turns=A + 4)) == ALIGN
    assert _append(lib, dm, rope=_rope(inter=2)) == INVALID
    assert _append(lib, dm, rope=_rope(scale=float("nan"))) == INVALID
    assert _append(lib, dm, qo=None) == INVALID and _append(lib, dm, q=None) == INVALID  # one without the other
    assert _passes(_append(lib, dm, q=None, qo=None))
    assert _append(lib, dm, k=None) == INVALID and _append(lib, dm, v=None) == INVALID
    assert _append(lib, dm, lens=None) == INVALID
    assert _append(lib, dm, no_kv=True) == INVALID  # k would go nowhere
    assert _passes(_append(lib, dm, no_kv=True, ko=A, kos=256, v=None, lens=None))
    assert _append(lib, dm, ko=A, kos=128) == SHAPE
    assert _append(lib, dm, qos=1020) == SHAPE and _append(lib, dm, qos=1028) == ALIGN


def test_append_in_place_keeps_the_strides(lib):
    dm = _dims()
    assert _append(lib, dm, qs=1024, qos=2048) == INVALID
    assert _passes(_append(lib, dm, qs=1024, qos=2048, qo=A + (1 << 20)))
    assert _append(lib, dm, ko=A, ks=256, kos=512) == INVALID
    assert _passes(_append(lib, dm, ko=A, ks=512, kos=512))


def test_struct_layouts():
    assert ctypes.sizeof(vpb.VpAttnDims) == 24
    assert ctypes.sizeof(vpb.VpPagedKv) == 3 * 8 + 3 * 4 + 4
    assert ctypes.sizeof(vpb.VpRopeOptions) == 8 + 3 * 4 + 4


def test_binding_refuses_before_the_library():
    with pytest.raises(ValueError):
        vpb.attn_dims(4, 2, 64, dtype=torch.float32)
    z = torch.zeros
    with pytest.raises(ValueError):  # a float32 cache
        vpb.paged_kv(z(2, 2, 16, 64), z(2, 2, 16, 64), z(1, 2, dtype=torch.int32))
    b = torch.bfloat16
    with pytest.raises(ValueError):  # k and v of different shapes
        vpb.paged_kv(z(2, 2, 16, 64, dtype=b), z(3, 2, 16, 64, dtype=b), z(1, 2, dtype=torch.int32))
    with pytest.raises(ValueError):  # a 64-bit table
        vpb.paged_kv(z(2, 2, 16, 64, dtype=b), z(2, 2, 16, 64, dtype=b), z(1, 2, dtype=torch.int64))
    with pytest.raises(ValueError):
        vpb.rope_options(z(8))
    for bad in (z(5, 4, 64), z(5, 3, 64, dtype=b), z(5, 4, 128, dtype=b), z(5, 4 * 64, dtype=b),
                z(5, 64, 4, dtype=b).transpose(1, 2), z(5, 8, 64, dtype=b)[:, ::2], z(5, 4, 64, dtype=torch.float16),
                z(5, 4, 64, dtype=b)):  # (the last: right but for living on the CPU)
        with pytest.raises(ValueError):
            vpb._rows_p(bad, (5, 4, 64), b)
    for bad in (z(3, dtype=torch.int64), z(4, dtype=torch.int32), z(3, dtype=torch.int32)):
        with pytest.raises(ValueError):
            vpb._ints_p(bad, 3, "cu")


# ---------------------------------------------------------------- rotary tables
def _freq(t):
    """Radians per position of a table."""
    return np.array([int(x) for x in t], np.float64) * (2 * math.pi / 2.0 ** 64)


def test_rope_turns():
    i = np.arange(32)
    f = 10000.0 ** (-2 * i / 64)
    assert np.allclose(_freq(vpb.rope_turns(64)), f, rtol=1e-15)
    assert np.allclose(_freq(vpb.rope_turns(64, base=500.0)), 500.0 ** (-2 * i / 64), rtol=1e-15)
    assert np.allclose(_freq(vpb.rope_turns(64, scaling="linear", factor=4.0)), f / 4, rtol=1e-15)
    grown = _freq(vpb.rope_turns(64, scaling="base", factor=8.0))
    assert np.isclose(grown[0], 1.0) and np.isclose(grown[-1], f[-1] / 8) and (np.diff(grown) < 0).all()
    parts = _freq(vpb.rope_turns(64, scaling="parts", factor=8.0, original_len=4096, low=1.0, high=32.0))
    made = 4096 * f / (2 * math.pi)  # turns within the original length
    assert np.allclose(parts[made >= 32], f[made >= 32]) and np.allclose(parts[made <= 1], f[made <= 1] / 8)
    mid = (made > 1) & (made < 32)
    assert mid.any() and ((parts[mid] < f[mid]) & (parts[mid] > f[mid] / 8)).all()
    assert vpb.rope_turns(0).numel() == 0
    for bad in (dict(rot_dim=7), dict(rot_dim=-2), dict(rot_dim=64, base=1.0), dict(rot_dim=64, factor=0.5),
                dict(rot_dim=64, scaling="other"), dict(rot_dim=64, scaling="parts", factor=2.0)):
        with pytest.raises(ValueError):
            vpb.rope_turns(**bad)


def test_turns_wrap_like_the_angle():
    """pos x turns, wrapped at 64 bits, is the angle modulo a turn."""
    turns = [int(x) for x in vpb.rope_turns(32)]
    for pos in (0, 1, 77, 2 ** 20 + 3, 2 ** 31 - 1):
        for i, t in enumerate(turns):
            angle = ((pos * t) % 2 ** 64) * (2 * math.pi / 2.0 ** 64)
            want = pos * 10000.0 ** (-2 * i / 32)
            assert abs(math.remainder(angle - want, 2 * math.pi)) < 2 ** -18

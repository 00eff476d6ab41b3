"""Argument checks of the streaming operators where calls are empty or addresses unaligned, without a
GPU."""
import pytest
import torch

from test_streaming_abi_cpu import A, ALIGN, BIG, INVALID, OK, SHAPE, _append, _dims, _kv, _passes, _paged, _prompt, _rope, lib  # noqa: F401

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses here are not real")


def test_no_tokens_need_no_addresses(lib):  # noqa: F811
    """Empty tensors have no address: T = 0 is nothing to do, whatever the pointers."""
    dm = _dims()
    for B in (0, 2):
        assert _prompt(lib, dm, T=0, B=B, q=None, k=None, v=None, cu=None, out=None, lse=None, ws=None, n=0) == OK
        assert _paged(lib, dm, T=0, B=B, q=None, cu=None, lens=None, out=None, lse=None, ws=None, n=0,
                      kv=_kv(None, None, None)) == OK
        assert _append(lib, dm, T=0, B=B, q=None, k=None, v=None, cu=None, lens=None, qo=None) == OK
    # what is no tensor is still checked
    assert _prompt(lib, _dims(d=32), T=0) == SHAPE and _paged(lib, _dims(dtype=2), T=0) == INVALID
    assert _append(lib, dm, T=0, no_rope=True) == INVALID and _append(lib, dm, T=0, rope=_rope(rot=24)) == SHAPE
    assert _append(lib, dm, T=0, B=-1) == INVALID


@pytest.mark.parametrize("off", [1, 2, 4, 8])
def test_append_workspace_alignment(lib, off):  # noqa: F811
    """The error word of a workspace at an odd address would be an unaligned atomic."""
    assert _append(lib, _dims(), ws=A + off, n=BIG) == ALIGN
    assert _passes(_append(lib, _dims(), ws=A, n=256))


@pytest.mark.parametrize("off", [1, 2, 3])
def test_alignment_of_32_bit_values(lib, off):  # noqa: F811
    """Lengths, offsets, positions, tables and log-sums are read and written as 32-bit values."""
    dm = _dims()
    for name in ("cu", "lse"):
        assert _prompt(lib, dm, **{name: A + off}) == ALIGN and _passes(_prompt(lib, dm, **{name: A + 4}))
    for name in ("cu", "lens", "lse"):
        assert _paged(lib, dm, **{name: A + off}) == ALIGN and _passes(_paged(lib, dm, **{name: A + 4}))
    for name in ("cu", "lens", "pos"):
        assert _append(lib, dm, **{name: A + off}) == ALIGN and _passes(_append(lib, dm, **{name: A + 4}))
    for call in (_paged, _append):
        assert call(lib, dm, kv=_kv(table=A + off)) == ALIGN and _passes(call(lib, dm, kv=_kv(table=A + 4)))

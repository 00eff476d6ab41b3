"""Argument checks of the streaming operators where calls are empty, without a GPU."""
import pytest
import torch

from test_streaming_abi_cpu import INVALID, OK, SHAPE, _append, _dims, _kv, _paged, _prompt, _rope, lib  # noqa: F401

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

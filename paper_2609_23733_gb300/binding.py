"""Thin ctypes binding of the C ABI in include/vp.h.

Functions carry the ABI's names and only marshal arguments: torch tensors become raw
device pointers, the current torch CUDA stream becomes the cudaStream_t, and a non-zero
vp_status raises VPError.  Every computation runs inside libvp.so; if the library is not
built (``__graft_entry__.build()``) the first call raises instead of falling back.
"""
from __future__ import annotations

import ctypes
import os
import math
from ctypes import POINTER, Structure, c_char_p, c_float, c_int32, c_int64, c_size_t, c_uint32, c_void_p

import numpy as np
import torch

from .build import LIB

VP_MODE_MEAN, VP_MODE_SURROGATE, VP_MODE_FULL = 0, 1, 2
VP_WS_ROUTER, VP_WS_LAYER, VP_WS_STACK, VP_WS_STACK_MERGE = 0, 1, 2, 3
VP_ACT_NONE, VP_ACT_GELU = 0, 1
VP_DEVERR_WAIT_TIMEOUT, VP_DEVERR_NAN_SALIENCY, VP_DEVERR_PAGE = 1, 2, 4
VP_VARIANT_MEAN_QPOOL, VP_VARIANT_MEAN_CONTEXT, VP_VARIANT_NO_RESIDUAL, VP_VARIANT_LINEAR_ATTENTION = 1, 2, 4, 8
KERNEL_CLASSES = ["gemm", "router_pool", "router_keys", "router_r", "bin_heads", "attn_full",
                  "surrogate", "mean", "layer_norm", "merge", "host_copy", "rope_append", "seq_attn"]

STATUS = {0: "VP_OK", 1: "VP_ERR_INVALID_ARG", 2: "VP_ERR_UNSUPPORTED_SHAPE", 3: "VP_ERR_ALIGNMENT",
          4: "VP_ERR_CUDA", 5: "VP_ERR_DEVICE_TIMEOUT", 6: "VP_ERR_WORKSPACE",
          7: "VP_ERR_UNSUPPORTED_DEVICE", 8: "VP_ERR_STATIC_SCRATCH"}


class VPError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)}")


class VpDims(Structure):
    _fields_ = [("N", c_int32), ("H", c_int32), ("d", c_int32), ("L", c_int32),
                ("tau_low", c_float), ("tau_high", c_float), ("variant", c_uint32)]


class VpRouterWeights(Structure):
    _fields_ = [(n, c_void_p) for n in ("W", "U", "w", "bW", "bU", "beta")]


class VpSurrogateWeights(Structure):
    _fields_ = [(n, c_void_p) for n in ("g1_w", "g1_b", "g2_w", "g2_b", "d1_w", "d1_b", "d2_w", "d2_b")]


class VpQkOptions(Structure):
    _fields_ = [(n, c_void_p) for n in ("q_norm_g", "q_norm_b", "k_norm_g", "k_norm_b")] + \
               [("norm_eps", c_float), ("rope", c_int32), ("tokens_per_view", c_int32),
                ("patch_start", c_int32), ("grid_w", c_int32), ("rope_base", c_float)]


class VpMergeOptions(Structure):
    _fields_ = [("stride", c_int32), ("tokens_per_view", c_int32), ("patch_start", c_int32),
                ("assign_out", c_void_p)]


class VpLayerWeights(Structure):
    _fields_ = [(n, c_void_p) for n in ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o", "ls1",
                                        "ln2_g", "ln2_b", "w_fc1", "b_fc1", "w_fc2", "b_fc2", "ls2")] + \
               [("router", VpRouterWeights), ("surrogate", VpSurrogateWeights),
                ("qk", POINTER(VpQkOptions)), ("merge", POINTER(VpMergeOptions))]


VP_DTYPES = {torch.bfloat16: 0, torch.float16: 1}


class VpAttnDims(Structure):
    _fields_ = [(n, c_int32) for n in ("Hq", "Hkv", "d", "dtype", "block")] + [("scale", c_float)]


class VpPagedKv(Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("page_table", c_void_p), ("n_pages", c_int32),
                ("page_size", c_int32), ("table_width", c_int32)]


class VpRopeOptions(Structure):
    _fields_ = [("turns", c_void_p), ("rot_dim", c_int32), ("interleaved", c_int32), ("scale", c_float)]


_lib = None

# (name, restype, argtypes)
_SIGS = [
    ("vp_status_string", c_char_p, [c_int32]),
    ("vp_workspace_size", c_int32, [POINTER(VpDims), c_int32, POINTER(c_size_t)]),
    ("vp_read_device_error", c_int32, [c_void_p, c_size_t, POINTER(c_uint32), c_void_p]),
    ("vp_selftest_wait_timeout", c_int32, [c_void_p, c_size_t, c_int64, c_void_p]),
    ("vp_router", c_int32, [POINTER(VpDims), c_void_p, POINTER(VpRouterWeights), c_void_p, c_void_p,
                            c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                            c_void_p]),
    ("vp_router_noalloc", c_int32, [POINTER(VpDims), c_void_p, POINTER(VpRouterWeights), c_void_p,
                                    c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                    c_void_p]),
    ("vp_router_noalloc_error", c_int32, [POINTER(c_uint32), c_void_p]),
    ("vp_bin_heads", c_int32, [c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                               c_void_p]),
    ("vp_head_attention", c_int32, [POINTER(VpDims), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                    POINTER(VpSurrogateWeights), c_void_p, c_void_p, c_void_p, c_size_t,
                                    c_void_p]),
    ("vp_linear", c_int32, [c_int32, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_int32, c_void_p,
                            c_void_p, c_void_p, c_void_p]),
    ("vp_layer_norm", c_int32, [c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_float, c_void_p,
                                c_void_p]),
    ("vp_moh_global_attention", c_int32, [POINTER(VpDims), c_void_p, c_void_p, c_void_p, c_void_p,
                                          c_void_p, POINTER(VpRouterWeights),
                                          POINTER(VpSurrogateWeights), POINTER(VpQkOptions), c_void_p,
                                          c_void_p, c_void_p,
                                          c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                          c_void_p]),
    ("vp_global_stack_host", c_int32, [POINTER(VpDims), c_int32, c_void_p, c_void_p, c_void_p,
                                       POINTER(VpLayerWeights), c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_float, c_void_p, c_size_t, c_void_p]),
    ("vp_attn_workspace_size", c_int32, [POINTER(VpAttnDims), c_int32, c_int32, POINTER(c_size_t)]),
    ("vp_rope_append", c_int32, [POINTER(VpAttnDims), POINTER(VpRopeOptions), c_int32, c_int32, c_void_p, c_int64,
                                 c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_void_p,
                                 POINTER(VpPagedKv), c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_size_t,
                                 c_void_p]),
    ("vp_prompt_attention", c_int32, [POINTER(VpAttnDims), c_int32, c_int32, c_void_p, c_int64, c_void_p, c_int64,
                                      c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_size_t,
                                      c_void_p]),
    ("vp_paged_attention", c_int32, [POINTER(VpAttnDims), c_int32, c_int32, c_void_p, c_int64, c_void_p, c_void_p,
                                     POINTER(VpPagedKv), c_void_p, c_int64, c_void_p, c_void_p, c_size_t, c_void_p]),
    ("vp_profile_begin", c_int32, [c_int32]),
    ("vp_profile_end", c_int32, [POINTER(c_int32), POINTER(c_int32), POINTER(c_float)]),
    ("vp_global_stack", c_int32, [POINTER(VpDims), c_int32, c_void_p, POINTER(VpLayerWeights),
                                  c_void_p, c_void_p, c_void_p, c_void_p, c_float, c_void_p, c_size_t,
                                  c_void_p]),
]
EXPORTS = [s[0] for s in _SIGS]


def lib():
    """Load libvp.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB):
            raise RuntimeError(f"{LIB} is missing: build it with __graft_entry__.build()")
        handle = ctypes.CDLL(LIB)
        for name, res, args in _SIGS:
            f = getattr(handle, name)
            f.restype = res
            f.argtypes = args
        _lib = handle
    return _lib


def _check(status: int, where: str):
    if status != 0:
        raise VPError(status, where)


def _p(t):
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        if t.device.type != "cuda":
            raise ValueError("device tensors are required (the library has no CPU path)")
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous")
        return t.data_ptr()
    return int(t)


def _host_p(t):
    """Address of a page-locked, contiguous CPU tensor (a host buffer the GPU can reach)."""
    if not isinstance(t, torch.Tensor) or t.device.type != "cpu":
        raise ValueError("a CPU tensor is required")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


# The current stream's handle without building a Stream object (a third of a short call's cost).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


if _raw_stream is None or _raw_device is None:
    _raw_stream, _raw_device = (lambda _: torch.cuda.current_stream().cuda_stream), (lambda: 0)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(_raw_device()) if torch.cuda.is_initialized() else torch.cuda.current_stream().cuda_stream


def _stream_of_tensors(stream):
    """_stream where device tensors are at hand (CUDA is up)."""
    return _raw_stream(_raw_device()) if stream is None else stream.cuda_stream


def dims(N, H=16, d=64, L=64, tau_low=0.01, tau_high=0.20, variant=0) -> VpDims:
    return VpDims(int(N), int(H), int(d), int(L), float(tau_low), float(tau_high), int(variant))


# The weight and option structs hold raw device addresses.  Each keeps a reference to the
# tensors it points into (``_keep``), so that a struct built from a temporary dict does not
# outlive its memory: a freed tensor's block is handed to the next allocation (a workspace,
# say), and the library would then read that as weights.  A struct copied into another one
# (``lw.router = ...``) or into a ctypes array does not carry the reference: the outer struct
# or the caller's list does.
def router_weights(w: dict) -> VpRouterWeights:
    rw = VpRouterWeights(_p(w["r_W"]), _p(w["r_U"]), _p(w["r_w"]), _p(w.get("r_bW")),
                         _p(w.get("r_bU")), _p(w.get("r_beta")))
    rw._keep = w
    return rw


def surrogate_weights(w: dict) -> VpSurrogateWeights:
    sw = VpSurrogateWeights(*[_p(w[k]) for k in ("s_g1_w", "s_g1_b", "s_g2_w", "s_g2_b",
                                                  "s_d1_w", "s_d1_b", "s_d2_w", "s_d2_b")])
    sw._keep = w
    return sw


def qk_options(w: dict = None, norm_eps: float = 1e-6, rope: bool = False, tokens_per_view: int = 1,
               patch_start: int = 0, grid_w: int = 1, rope_base: float = 100.0) -> VpQkOptions:
    """vp_qk_options from device tensors w["q_norm_g"], ... (each pair optional) and the
    RoPE token layout."""
    w = w or {}
    o = VpQkOptions(*[_p(w.get(k)) for k in ("q_norm_g", "q_norm_b", "k_norm_g", "k_norm_b")])
    o.norm_eps = norm_eps
    o.rope = 1 if rope else 0
    o.tokens_per_view = tokens_per_view
    o.patch_start = patch_start
    o.grid_w = grid_w
    o.rope_base = rope_base
    o._keep = w
    return o


def merge_options(stride: int, tokens_per_view: int, patch_start: int = 5, assign_out=None) -> VpMergeOptions:
    """vp_merge_options; assign_out: int32 device tensor [N] or None."""
    mo = VpMergeOptions(stride, tokens_per_view, patch_start, _p(assign_out))
    mo._keep = assign_out
    return mo


def layer_weights(w: dict, qk: VpQkOptions = None, merge: VpMergeOptions = None) -> VpLayerWeights:
    lw = VpLayerWeights(*[_p(w[k]) for k in ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o", "ls1",
                                             "ln2_g", "ln2_b", "w_fc1", "b_fc1", "w_fc2", "b_fc2",
                                             "ls2")])
    lw.router = router_weights(w)
    lw.surrogate = surrogate_weights(w)
    lw._keep = w
    if qk is not None:
        lw.qk = ctypes.pointer(qk)
        lw._qk_keep = qk  # the struct must outlive the call
    if merge is not None:
        lw.merge = ctypes.pointer(merge)
        lw._merge_keep = merge
    return lw


def attn_dims(Hq, Hkv=None, d=64, dtype=torch.bfloat16, block=1, scale=None) -> VpAttnDims:
    """vp_attn_dims of the streaming operators; scale None: 1 / sqrt(d)."""
    if dtype not in VP_DTYPES:
        raise ValueError("dtype must be torch.bfloat16 or torch.float16")
    return VpAttnDims(int(Hq), int(Hq if Hkv is None else Hkv), int(d), VP_DTYPES[dtype], int(block),
                      1.0 / math.sqrt(d) if scale is None else float(scale))


def paged_kv(k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor) -> VpPagedKv:
    """vp_paged_kv of a cache: k, v [n_pages][Hkv][page_size][d], page_table [B][width] int32."""
    if k.dim() != 4 or v.shape != k.shape or v.dtype != k.dtype or k.dtype not in VP_DTYPES:
        raise ValueError("k and v: one 16-bit type and one shape [n_pages][Hkv][page_size][d]")
    if page_table.dim() != 2 or page_table.dtype != torch.int32:
        raise ValueError("page_table: int32 [sequences][pages of a sequence]")
    o = VpPagedKv(_p(k), _p(v), _p(page_table), k.shape[0], k.shape[2], page_table.shape[1])
    o._keep = (k, v, page_table)
    o._heads = (k.shape[1], k.shape[3], VP_DTYPES[k.dtype])
    o._rows = page_table.shape[0]
    return o


def rope_turns(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
               original_len: int = 0, low: float = 1.0, high: float = 32.0) -> torch.Tensor:
    """The table of vp_rope_options: turns per position of each of the rot_dim / 2 pairs, as 64-bit
    fractions of a turn (int64, on the CPU).  Pair i turns by base^(-2 i / rot_dim) radians per
    position.  For contexts longer than the original_len positions of the training, by ``factor``:
      "linear"  every frequency divided by factor (positions interpolated)
      "base"    the base raised by factor^(rot_dim / (rot_dim - 2)): the slowest pair is divided by
                factor, the fastest kept
      "parts"   by the turns a pair makes within original_len: divided by factor below ``low`` turns,
                kept above ``high``, mixed linearly in between
    """
    if rot_dim < 0 or rot_dim % 2 or not base > 1 or not factor >= 1:
        raise ValueError("rot_dim must be even, base > 1 and factor >= 1")
    if scaling not in ("none", "linear", "base", "parts"):
        raise ValueError(f"unknown scaling {scaling!r}")
    if scaling == "parts" and (original_len < 1 or not high > low):
        raise ValueError("scaling 'parts' needs original_len >= 1 and high > low")
    if scaling == "base" and rot_dim > 2:
        base = base * factor ** (rot_dim / (rot_dim - 2))
    turns = []
    for i in range(rot_dim // 2):
        f = base ** (-2.0 * i / rot_dim) / (2 * math.pi)
        if scaling == "linear":
            f /= factor
        elif scaling == "parts":
            keep = min(1.0, max(0.0, (original_len * f - low) / (high - low)))
            f = f * (keep + (1 - keep) / factor)
        turns.append(int(f * 2.0 ** 64))
    return torch.tensor(turns, dtype=torch.int64)


def rope_options(turns: torch.Tensor, interleaved: bool = False, scale: float = 1.0) -> VpRopeOptions:
    """vp_rope_options from the device table of ``rope_turns`` (int64 [rot_dim / 2])."""
    if turns.dtype != torch.int64 or turns.dim() != 1:
        raise ValueError("turns: int64 [rot_dim / 2]")
    o = VpRopeOptions(_p(turns) if turns.numel() else None, 2 * turns.numel(), 1 if interleaved else 0, float(scale))
    o._keep = turns
    return o


def to_device(w: dict, device="cuda") -> dict:
    """Upload a parameter dict from ``synth`` (bf16 bits as uint16, fp32 arrays)."""
    out = {}
    for k, v in w.items():
        v = np.ascontiguousarray(v)
        t = torch.from_numpy(v.view(np.int16)).view(torch.bfloat16) if v.dtype == np.uint16 else torch.from_numpy(v)
        out[k] = t.to(device)
    return out


def bf16_from_bits(u, device="cuda") -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(u).view(np.int16)).view(torch.bfloat16).to(device)


def bits_from_bf16(t: torch.Tensor) -> np.ndarray:
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


# ---------------------------------------------------------------- ABI wrappers
def vp_status_string(status: int) -> str:
    return lib().vp_status_string(int(status)).decode()


def vp_workspace_size(dm: VpDims, what: int) -> int:
    n = c_size_t(0)
    _check(lib().vp_workspace_size(ctypes.byref(dm), int(what), ctypes.byref(n)), "vp_workspace_size")
    return n.value


def workspace(dm: VpDims, what: int, device="cuda") -> torch.Tensor:
    """A zeroed device workspace of the size the library asks for."""
    return torch.zeros(vp_workspace_size(dm, what), dtype=torch.uint8, device=device)


def vp_selftest_wait_timeout(ws: torch.Tensor, limit_ns: int, stream=None):
    """Enqueues the library's bounded-wait self-test: a wait that nothing satisfies gives up
    after limit_ns and sets the timeout bit of ws's error word."""
    _check(lib().vp_selftest_wait_timeout(_p(ws), ws.numel(), int(limit_ns), _stream(stream)),
           "vp_selftest_wait_timeout")


def vp_read_device_error(ws: torch.Tensor, stream=None) -> int:
    bits = c_uint32(0)
    st = lib().vp_read_device_error(_p(ws), ws.numel(), ctypes.byref(bits), _stream(stream))
    if st not in (0, 5):
        _check(st, "vp_read_device_error")
    return bits.value


def vp_router(dm, qkv, rw: VpRouterWeights, force_modes, s, modes, q_pool, ctx, mean_v, r, ws, stream=None):
    _check(lib().vp_router(ctypes.byref(dm), _p(qkv), ctypes.byref(rw), _p(force_modes), _p(s), _p(modes),
                           _p(q_pool), _p(ctx), _p(mean_v), _p(r), _p(ws), ws.numel(), _stream(stream)),
           "vp_router")


def vp_router_noalloc(dm, qkv, rw: VpRouterWeights, force_modes, s, modes, q_pool, ctx, mean_v, r,
                      stream=None):
    """vp_router without a workspace: scratch comes from a fixed buffer inside the library,
    for callers that cannot allocate device memory (see include/vp.h)."""
    _check(lib().vp_router_noalloc(ctypes.byref(dm), _p(qkv), ctypes.byref(rw), _p(force_modes), _p(s),
                                   _p(modes), _p(q_pool), _p(ctx), _p(mean_v), _p(r), _stream(stream)),
           "vp_router_noalloc")


def vp_router_noalloc_error(stream=None) -> int:
    """Reads and clears the device error bits of vp_router_noalloc's fixed buffer."""
    bits = c_uint32(0)
    st = lib().vp_router_noalloc_error(ctypes.byref(bits), _stream(stream))
    if st not in (0, 5):
        _check(st, "vp_router_noalloc_error")
    return bits.value


def vp_bin_heads(H, N, modes, head_ids, offsets, work=None, n_work=None, stream=None):
    _check(lib().vp_bin_heads(int(H), int(N), _p(modes), _p(head_ids), _p(offsets), _p(work), _p(n_work),
                              _stream(stream)), "vp_bin_heads")


def vp_head_attention(dm, qkv, head_ids, offsets, ctx, mean_v, sw: VpSurrogateWeights, y, ws, stream=None,
                      s_attn=None):
    _check(lib().vp_head_attention(ctypes.byref(dm), _p(qkv), _p(head_ids), _p(offsets), _p(ctx), _p(mean_v),
                                   ctypes.byref(sw), _p(y), _p(s_attn), _p(ws), ws.numel(), _stream(stream)),
           "vp_head_attention")


def vp_linear(A, W, bias=None, act=VP_ACT_NONE, scale=None, residual=None, out=None, stream=None):
    M, K = A.shape
    Nout = W.shape[0]
    if out is None:
        out = torch.empty((M, Nout), dtype=torch.bfloat16, device=A.device)
    _check(lib().vp_linear(M, Nout, K, _p(A), _p(W), _p(bias), int(act), _p(scale), _p(residual), _p(out),
                           _stream(stream)), "vp_linear")
    return out


def vp_layer_norm(x, gamma, beta, eps=1e-6, out=None, stream=None):
    M, D = x.shape
    if out is None:
        out = torch.empty_like(x)
    _check(lib().vp_layer_norm(M, D, _p(x), _p(gamma), _p(beta), float(eps), _p(out), _stream(stream)),
           "vp_layer_norm")
    return out


def vp_moh_global_attention(dm, x, w_qkv, b_qkv, w_o, b_o, rw, sw, force_modes, out, qkv_out, y_out,
                            s_out, modes_out, ws, stream=None, s_attn_out=None, qk=None):
    _check(lib().vp_moh_global_attention(ctypes.byref(dm), _p(x), _p(w_qkv), _p(b_qkv), _p(w_o), _p(b_o),
                                         ctypes.byref(rw), ctypes.byref(sw),
                                         ctypes.byref(qk) if qk is not None else None,
                                         _p(force_modes), _p(out),
                                         _p(qkv_out), _p(y_out), _p(s_out), _p(s_attn_out), _p(modes_out),
                                         _p(ws), ws.numel(), _stream(stream)), "vp_moh_global_attention")


def vp_global_stack(dm, x_inout, layers, force_modes, modes_out, s_out, ln_eps, ws, stream=None,
                    s_attn_out=None):
    arr = (VpLayerWeights * len(layers))(*layers)
    _check(lib().vp_global_stack(ctypes.byref(dm), len(layers), _p(x_inout), arr, _p(force_modes),
                                 _p(modes_out), _p(s_out), _p(s_attn_out), float(ln_eps), _p(ws), ws.numel(),
                                 _stream(stream)), "vp_global_stack")


def vp_global_stack_host(dm, x_in, x_out, x_dev, layers, force_modes, modes_out, s_out, ln_eps, ws,
                         stream=None, s_attn_out=None):
    """vp_global_stack on tokens in page-locked host memory (x_in, x_out: pinned CPU tensors);
    x_dev is the device buffer the blocks run on."""
    arr = (VpLayerWeights * len(layers))(*layers)
    _check(lib().vp_global_stack_host(ctypes.byref(dm), len(layers), _host_p(x_in), _host_p(x_out), _p(x_dev), arr,
                                      _p(force_modes), _p(modes_out), _p(s_out), _p(s_attn_out), float(ln_eps),
                                      _p(ws), ws.numel(), _stream(stream)), "vp_global_stack_host")


def vp_attn_workspace_size(dims: VpAttnDims, T: int, B: int) -> int:
    n = c_size_t(0)
    _check(lib().vp_attn_workspace_size(ctypes.byref(dims), int(T), int(B), ctypes.byref(n)),
           "vp_attn_workspace_size")
    return n.value


def attn_workspace(dims: VpAttnDims, T: int, B: int, device="cuda") -> torch.Tensor:
    """A device workspace for up to T packed tokens in up to B sequences, its error word zero."""
    ws = torch.empty(vp_attn_workspace_size(dims, T, B), dtype=torch.uint8, device=device)
    ws[:256].zero_()
    return ws


_byref = ctypes.byref
_TORCH_DTYPES = {v: k for k, v in VP_DTYPES.items()}


def _rows_p(t, shape, dtype):
    """(address, token stride) of a [T][heads][d] device tensor whose heads and channels are contiguous."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype is not dtype or not t.is_cuda:
        raise ValueError(f"expected a device tensor {list(shape)} of {dtype}, got {list(t.shape)} of {t.dtype} on "
                         f"{t.device}")
    T, heads, d = shape
    s0, s1, s2 = t.stride()
    if s2 != 1 or (s1 != d and heads > 1):
        raise ValueError("heads and channels must be contiguous")
    # a single token has no stride of its own: any legal one stands for it
    return t.data_ptr(), s0 if T > 1 else heads * d


def _ints_p(t, n, what):
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.numel() != n or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous int32 device tensor with {n} values")
    return t.data_ptr()


def _kv_ref(kv, dims, B):
    if kv is None:
        return None
    if kv._heads != (dims.Hkv, dims.d, dims.dtype):
        raise ValueError("the cache's heads, head dim or type are not those of dims")
    if kv._rows < B:
        raise ValueError(f"the page table has {kv._rows} rows for {B} sequences")
    return _byref(kv)


def vp_rope_append(dims: VpAttnDims, rope: VpRopeOptions, q, k, v, cu, kv_len, positions, kv: VpPagedKv = None,
                   q_out=None, k_out=None, ws=None, stream=None):
    """Rotates q into q_out and k into the cache (and / or k_out), and writes v to the cache."""
    T, B, d, dt = k.shape[0], cu.numel() - 1, dims.d, _TORCH_DTYPES.get(dims.dtype)
    q_shape, kv_shape = (T, dims.Hq, d), (T, dims.Hkv, d)
    qp, qs = _rows_p(q, q_shape, dt)
    kp, ks = _rows_p(k, kv_shape, dt)
    vp, vs = _rows_p(v, kv_shape, dt)
    qo, qos = _rows_p(q_out, q_shape, dt)
    ko, kos = _rows_p(k_out, kv_shape, dt)
    wp, wn = (None, 0) if ws is None else _ws_p(ws)
    st = lib().vp_rope_append(_byref(dims), _byref(rope), T, B, qp, qs, kp, ks, vp, vs, _ints_p(cu, B + 1, "cu"),
                              _ints_p(kv_len, B, "kv_len"), _ints_p(positions, T, "positions"), _kv_ref(kv, dims, B),
                              qo, qos, ko, kos, wp, wn, _stream_of_tensors(stream))
    if st:
        raise VPError(st, "vp_rope_append")


def _ws_p(ws):
    if not ws.is_cuda or not ws.is_contiguous() or ws.dtype is not torch.uint8:
        raise ValueError("ws: a contiguous uint8 device tensor (attn_workspace)")
    return ws.data_ptr(), ws.numel()


def _lse_p(lse, T, dims):
    if lse is None:
        return None
    if lse.dtype is not torch.float32 or lse.numel() != T * dims.Hq or not lse.is_cuda or not lse.is_contiguous():
        raise ValueError(f"lse: a contiguous float32 device tensor [{T}][{dims.Hq}]")
    return lse.data_ptr()


def vp_prompt_attention(dims: VpAttnDims, q, k, v, cu, out, lse, ws, stream=None):
    """Softmax attention of whole packed prompts over themselves: q, k, v, out [T][heads][d], cu int32 [B + 1],
    lse float32 [T][Hq] or None, ws from ``attn_workspace``."""
    T, B, d, dt = q.shape[0], cu.numel() - 1, dims.d, _TORCH_DTYPES.get(dims.dtype)
    q_shape, kv_shape = (T, dims.Hq, d), (T, dims.Hkv, d)
    qp, qs = _rows_p(q, q_shape, dt)
    kp, ks = _rows_p(k, kv_shape, dt)
    vp, vs = _rows_p(v, kv_shape, dt)
    op, os_ = _rows_p(out, q_shape, dt)
    st = lib().vp_prompt_attention(_byref(dims), T, B, qp, qs, kp, ks, vp, vs, _ints_p(cu, B + 1, "cu"), op,
                                   os_, _lse_p(lse, T, dims), *_ws_p(ws), _stream_of_tensors(stream))
    if st:
        raise VPError(st, "vp_prompt_attention")


def vp_paged_attention(dims: VpAttnDims, q, cu, kv_len, kv: VpPagedKv, out, lse, ws, stream=None):
    """Softmax attention of new tokens (chunks or single tokens, already appended) over the paged cache; kv_len
    int32 [B] counts them in.  The rest as in ``vp_prompt_attention``."""
    T, B = q.shape[0], cu.numel() - 1
    shape, dt = (T, dims.Hq, dims.d), _TORCH_DTYPES.get(dims.dtype)
    qp, qs = _rows_p(q, shape, dt)
    op, os_ = _rows_p(out, shape, dt)
    st = lib().vp_paged_attention(_byref(dims), T, B, qp, qs, _ints_p(cu, B + 1, "cu"),
                                  _ints_p(kv_len, B, "kv_len"), _kv_ref(kv, dims, B), op, os_,
                                  _lse_p(lse, T, dims), *_ws_p(ws), _stream_of_tensors(stream))
    if st:
        raise VPError(st, "vp_paged_attention")


def vp_profile_begin(max_launches: int):
    _check(lib().vp_profile_begin(int(max_launches)), "vp_profile_begin")


def vp_profile_end():
    """Returns (total launches, {class: launches}, {class: summed ms})."""
    n = c_int32(0)
    cnt = (c_int32 * len(KERNEL_CLASSES))()
    ms = (c_float * len(KERNEL_CLASSES))()
    _check(lib().vp_profile_end(ctypes.byref(n), cnt, ms), "vp_profile_end")
    return n.value, dict(zip(KERNEL_CLASSES, list(cnt))), dict(zip(KERNEL_CLASSES, list(ms)))

"""Python binding of librmuscle.so, the Action Cache sparse-FFN hot path for MI355X (gfx950).

Argument marshalling only: every function checks tensor devices, dtypes and shapes, turns them into raw
device pointers plus the current HIP stream, and calls the C ABI function of the same name (declared in
include/rmuscle.h).  All computation runs in the library's HIP kernels; there is no fallback.  If the library
is not built, or no GPU is present, the calls raise.

Layouts (see include/rmuscle.h for the full contract):
  mask  uint8/bool [N][d_ff] -> idx int32 [N][d_ff] (ascending, -1 tail), count int32 [N]
  x, y  float32 [B][T][d];  weights [d_ff][d] float32 or bfloat16, row n = neuron n (w_down neuron-major)
  idx   int32 [B][d_ff] per layer ([L][B][d_ff] for a stack), count int32 [B] ([L][B])
  Eq. 4 anchor state: y_anchor float32 [L][B][T][d], h_anchor float32 [L][B][max_count][T]
  attention: q, out [B][T][n_q_heads][D], k, v [B][N][n_kv_heads][D], float32 or bfloat16, any strides whose last
  is 1; span int32 [B][T][2]
  paged caches: [n_pages][page][n_kv_heads][D], float32 or bfloat16, any strides whose last is 1; table int32
  [n_seqs][max_pages]
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
from typing import Optional, Sequence, Tuple

import torch

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
# The in-tree build; RMUSCLE_LIB may name another build of the same library (e.g. for A/B timing).
LIB_PATH = os.environ.get("RMUSCLE_LIB") or os.path.join(PKG_DIR, "librmuscle.so")

NOALLOC_SCRATCH_BYTES = 32 << 20  # RM_NOALLOC_SCRATCH_BYTES

RM_OK = 0
RM_ERR_INVALID_ARG = -1
RM_ERR_SHAPE = -2
RM_ERR_DTYPE = -3
RM_ERR_ALIGN = -4
RM_ERR_WORKSPACE = -5
RM_ERR_HIP = -6

RM_F32 = 0
RM_BF16 = 1
RM_ACT_SILU = 0
RM_ACT_GELU_TANH = 1
ACTS = {"silu": RM_ACT_SILU, "gelu_tanh": RM_ACT_GELU_TANH}
RM_KERNEL_GATEUP = 0
RM_KERNEL_DOWN = 1
RM_KERNEL_SCORES = 2
RM_KERNEL_GROUP_SELECT = 3
RM_KERNEL_LAYER = 4

EXPORTED = ("rm_mask_compact", "rm_workspace_size", "rm_sparse_ffn_layer", "rm_sparse_ffn_layer_noalloc",
            "rm_sparse_ffn_stack",
            "rm_masked_ffn_layer", "rm_masked_ffn_stack", "rm_dense_ffn_ref", "rm_anchor_ffn_stack",
            "rm_delta_ffn_stack", "rm_gather_stack_rows", "rm_context_select", "rm_context_workspace_size",
            "rm_context_ffn", "rm_context_pack_size", "rm_context_pack", "rm_context_ffn_packed", "rm_neuron_norms",
            "rm_group_masks",
            "rm_qk_norm_rope", "rm_attn_spans", "rm_span_attention_workspace_size", "rm_span_attention",
            "rm_prefix_attention_workspace_size", "rm_prefix_attention",
            "rm_page_slots", "rm_paged_attention_workspace_size", "rm_paged_attention", "rm_block_norm",
            "rm_profile_kernel_events", "rm_layer_kernels", "rm_stream_read",
            "rm_status_string", "rm_last_error")

# (w_gate, w_up, w_down, norm_g) or (w_gate, w_up, w_down, norm_g, out_gate); norm_g and out_gate may be None.
Layer = Tuple[Optional[torch.Tensor], ...]


class RmError(RuntimeError):
    def __init__(self, status: int, detail: str):
        self.status = status
        self.detail = detail
        super().__init__(f"{status_string(status)}: {detail}")


class FfnShape(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("d_ff", ctypes.c_int32), ("wdtype", ctypes.c_int32),
                ("norm_eps", ctypes.c_float), ("act", ctypes.c_int32)]


class LayerWeights(ctypes.Structure):
    _fields_ = [("w_gate", ctypes.c_void_p), ("w_up", ctypes.c_void_p), ("w_down", ctypes.c_void_p),
                ("norm_g", ctypes.c_void_p), ("out_gate", ctypes.c_void_p)]


class Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64),
                ("head", ctypes.c_int64)]


class AttnShape(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("softcap", ctypes.c_float)]


_lib: Optional[ctypes.CDLL] = None


def library_path() -> str:
    return LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load librmuscle.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built: run `python -m paper_2609_19104_amd.build` "
                           "(or __graft_entry__.build()) first")
    lib = ctypes.CDLL(LIB_PATH)
    i32, i64, vp, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
    sp, wp = ctypes.POINTER(FfnShape), ctypes.POINTER(LayerWeights)
    f32 = ctypes.c_float
    sigs = {
        "rm_mask_compact": [vp, i32, i32, vp, vp, vp],
        "rm_workspace_size": [sp, i32, i32, i32, ctypes.POINTER(sz)],
        "rm_sparse_ffn_layer": [sp, wp, i32, i32, vp, vp, vp, vp, i32, vp, sz, vp],
        "rm_sparse_ffn_layer_noalloc": [sp, wp, i32, i32, vp, vp, vp, vp, i32, vp],
        "rm_sparse_ffn_stack": [sp, wp, i32, i32, i32, vp, vp, vp, vp, i32, vp, sz, vp],
        "rm_masked_ffn_layer": [sp, wp, i32, i32, vp, vp, vp, vp, vp, i32, vp, sz, vp],
        "rm_masked_ffn_stack": [sp, wp, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp, sz, vp],
        "rm_dense_ffn_ref": [sp, wp, i32, i32, vp, vp, vp, sz, vp],
        "rm_anchor_ffn_stack": [sp, wp, i32, i32, i32, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp],
        "rm_delta_ffn_stack": [sp, wp, i32, i32, i32, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp],
        "rm_gather_stack_rows": [sp, wp, i32, vp, vp, i32, vp, vp],
        "rm_context_select": [vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp],
        "rm_context_workspace_size": [sp, i32, i32, ctypes.POINTER(sz)],
        "rm_context_ffn": [sp, vp, vp, vp, i32, vp, vp, vp, i32, vp, vp, sz, vp],
        "rm_context_pack_size": [sp, ctypes.POINTER(sz)],
        "rm_context_pack": [sp, vp, vp, vp, vp, sz, vp],
        "rm_context_ffn_packed": [sp, vp, i32, vp, vp, vp, i32, vp, vp, sz, vp],
        "rm_neuron_norms": [vp, i32, i32, i32, vp, vp],
        "rm_group_masks": [vp, i32, i32, i32, i32, vp, i32, vp, vp, vp],
        "rm_qk_norm_rope": [i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, i32, i32, vp, vp,
                            f32, vp],
        "rm_attn_spans": [i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp],
        "rm_span_attention_workspace_size": [vp, i32, i32, i32, ctypes.POINTER(sz)],
        "rm_span_attention": [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
        "rm_prefix_attention_workspace_size": [vp, i32, i32, i32, i32, i32, ctypes.POINTER(sz)],
        "rm_prefix_attention": [vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp],
        "rm_page_slots": [i32] * 5 + [vp] * 14,
        "rm_paged_attention_workspace_size": [vp, i32, i32, i32, ctypes.POINTER(sz)],
        "rm_paged_attention": [vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp],
        "rm_block_norm": [i32, i32, i32, i32, i32, i32, vp, vp, i32, vp, vp, i64, f32, f32, vp, vp, vp, i64, vp, i64, f32,
                          vp, vp],
        "rm_profile_kernel_events": [i32, vp, vp],
        "rm_layer_kernels": [sp, i32, i32, i32, ctypes.POINTER(ctypes.c_uint32)],
        "rm_stream_read": [vp, sz, i32, vp, vp],
        "rm_status_string": [i32],
        "rm_last_error": [],
    }
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_char_p if name in ("rm_status_string", "rm_last_error") else ctypes.c_int
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().rm_status_string(status).decode()


def last_error() -> str:
    return load_library().rm_last_error().decode()


def _check(status: int) -> None:
    if status != RM_OK:
        raise RmError(status, last_error())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _no_gpu(*_) -> int:
    raise RuntimeError("this build of torch has no GPU support")


# (A torch without a GPU has neither; what needs none, such as workspace sizes, works there.)
_current_device = getattr(torch._C, "_cuda_getDevice", _no_gpu)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _no_gpu)


def _stream(stream) -> Optional[int]:
    if stream is None:  # the current stream's handle itself, without a Stream object around it
        return _raw_stream(_current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _need_cuda(name: str, t: torch.Tensor, dtypes, ndim: Optional[int] = None) -> None:
    # Every tensor of every call comes through here (a stack's weights alone are 54): the usual case in one test, the
    # reason only when it fails.
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.is_contiguous()
            and (ndim is None or t.dim() == ndim)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on a HIP device, got {t.device}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got {tuple(t.shape)}")


def wdtype_of(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return RM_BF16
    if t.dtype == torch.float32:
        return RM_F32
    raise ValueError(f"weights must be float32 or bfloat16, got {t.dtype}")


def _shape(layer: Layer, eps: float, act: str = "silu") -> FfnShape:
    wg = layer[0]
    if act not in ACTS:
        raise ValueError(f"act must be one of {sorted(ACTS)}, got {act!r}")
    return FfnShape(int(wg.shape[1]), int(wg.shape[0]), wdtype_of(wg), float(eps), ACTS[act])


def _weights(layer: Layer, B: Optional[int] = None) -> LayerWeights:
    if len(layer) not in (4, 5):
        raise ValueError("a layer is (w_gate, w_up, w_down, norm_g[, out_gate])")
    wg, wu, wd, g = layer[:4]
    gate = layer[4] if len(layer) == 5 else None
    full = wg.shape
    d_ff, d = full
    for name, w in (("w_gate", wg), ("w_up", wu), ("w_down", wd)):
        _need_cuda(name, w, (wg.dtype,), 2)
        if w.shape != full:
            raise ValueError(f"{name} has shape {tuple(w.shape)}, expected {(d_ff, d)} (neuron-major)")
    if g is not None:
        _need_cuda("norm_g", g, (torch.float32,), 1)
        if g.shape[0] != d:
            raise ValueError("norm_g must have d entries")
    if gate is not None:
        _need_cuda("out_gate", gate, (torch.float32,))
        if B is not None and gate.numel() != B * d:
            raise ValueError(f"out_gate must be [B][d] = [{B}][{d}]")
    return LayerWeights(wg.data_ptr(), wu.data_ptr(), wd.data_ptr(), _ptr(g), _ptr(gate))


def _activations(x: torch.Tensor, y: torch.Tensor, d: int) -> Tuple[int, int]:
    _need_cuda("x", x, (torch.float32,), 3)
    _need_cuda("y", y, (torch.float32,), 3)
    if x.shape != y.shape or x.shape[2] != d:
        raise ValueError(f"x {tuple(x.shape)} and y {tuple(y.shape)} must both be [B][T][{d}]")
    return int(x.shape[0]), int(x.shape[1])


# ----------------------------------------------------------------------------------------------------------
# The C ABI calls
# ----------------------------------------------------------------------------------------------------------

def rm_mask_compact(mask: torch.Tensor, idx: torch.Tensor, count: torch.Tensor, stream=None) -> None:
    """mask uint8/bool [N][d_ff] -> idx int32 [N][d_ff] (ascending, -1 tail) and count int32 [N]."""
    _need_cuda("mask", mask, (torch.uint8, torch.bool), 2)
    n, d_ff = mask.shape
    _need_cuda("idx", idx, (torch.int32,))
    _need_cuda("count", count, (torch.int32,))
    if idx.numel() != n * d_ff or count.numel() != n:
        raise ValueError("idx must hold N*d_ff and count N entries")
    _check(load_library().rm_mask_compact(mask.data_ptr(), n, d_ff, idx.data_ptr(), count.data_ptr(),
                                          _stream(stream)))


def rm_workspace_size(d: int, d_ff: int, wdtype: int, B: int, T: int, max_count: int, eps: float = 1e-6) -> int:
    out = ctypes.c_size_t(0)
    shape = FfnShape(d, d_ff, wdtype, eps)
    _check(load_library().rm_workspace_size(ctypes.byref(shape), B, T, max_count, ctypes.byref(out)))
    return int(out.value)


def rm_layer_kernels(d: int, d_ff: int, wdtype: int, B: int, T: int, max_count: int, eps: float = 1e-6) -> int:
    """Bit mask of the RM_KERNEL_* ids a single-layer call of this shape launches on the current device."""
    out = ctypes.c_uint32(0)
    shape = FfnShape(d, d_ff, wdtype, eps)
    _check(load_library().rm_layer_kernels(ctypes.byref(shape), B, T, max_count, ctypes.byref(out)))
    return int(out.value)


def workspace(d: int, d_ff: int, wdtype: int, B: int, T: int, max_count: int, device="cuda") -> torch.Tensor:
    """Allocate a workspace tensor (uint8) of the size rm_workspace_size asks for."""
    return torch.empty(rm_workspace_size(d, d_ff, wdtype, B, T, max_count), dtype=torch.uint8, device=device)


def _ws(ws: torch.Tensor) -> Tuple[int, int]:
    _need_cuda("ws", ws, (torch.uint8,))
    return ws.data_ptr(), ws.numel()


def rm_sparse_ffn_layer(x: torch.Tensor, y: torch.Tensor, layer: Layer, idx: torch.Tensor, count: torch.Tensor,
                        max_count: int, ws: torch.Tensor, eps: float = 1e-6, act: str = "silu", stream=None) -> None:
    """y = x + masked GLU FFN over the listed neurons (y may be x); act "silu" (SwiGLU) or "gelu_tanh" (GeGLU)."""
    shape = _shape(layer, eps, act)
    B, T = _activations(x, y, shape.d)
    w = _weights(layer, B)
    _need_cuda("idx", idx, (torch.int32,))
    _need_cuda("count", count, (torch.int32,))
    if idx.numel() != B * shape.d_ff or count.numel() != B:
        raise ValueError("idx must be [B][d_ff] and count [B]")
    wp, wn = _ws(ws)
    _check(load_library().rm_sparse_ffn_layer(ctypes.byref(shape), ctypes.byref(w), B, T, x.data_ptr(),
                                              y.data_ptr(), idx.data_ptr(), count.data_ptr(), int(max_count),
                                              wp, wn, _stream(stream)))


def rm_sparse_ffn_layer_noalloc(x: torch.Tensor, y: torch.Tensor, layer: Layer, idx: torch.Tensor,
                                count: torch.Tensor, max_count: int, eps: float = 1e-6, act: str = "silu",
                                stream=None) -> None:
    """rm_sparse_ffn_layer with the library's own per-device scratch instead of a workspace (no allocation; calls
    that may overlap on one GPU must be ordered by the caller)."""
    shape = _shape(layer, eps, act)
    B, T = _activations(x, y, shape.d)
    w = _weights(layer, B)
    _need_cuda("idx", idx, (torch.int32,))
    _need_cuda("count", count, (torch.int32,))
    if idx.numel() != B * shape.d_ff or count.numel() != B:
        raise ValueError("idx must be [B][d_ff] and count [B]")
    _check(load_library().rm_sparse_ffn_layer_noalloc(ctypes.byref(shape), ctypes.byref(w), B, T, x.data_ptr(),
                                                      y.data_ptr(), idx.data_ptr(), count.data_ptr(),
                                                      int(max_count), _stream(stream)))


def _stack_args(x: torch.Tensor, y: torch.Tensor, layers: Sequence[Layer], idx: torch.Tensor,
                count: torch.Tensor, eps: float, act: str):
    L = len(layers)
    if L == 0:
        raise ValueError("at least one layer")
    shape = _shape(layers[0], eps, act)
    B, T = _activations(x, y, shape.d)
    arr = (LayerWeights * L)()
    for l, layer in enumerate(layers):
        s = _shape(layer, eps, act)
        if (s.d, s.d_ff, s.wdtype) != (shape.d, shape.d_ff, shape.wdtype):
            raise ValueError("every layer of a stack must have the same shape and dtype")
        arr[l] = _weights(layer, B)
    _need_cuda("idx", idx, (torch.int32,))
    _need_cuda("count", count, (torch.int32,))
    if idx.numel() != L * B * shape.d_ff or count.numel() != L * B:
        raise ValueError("idx must be [L][B][d_ff] and count [L][B]")
    return shape, arr, L, B, T


def _anchor_state(y_anchor: torch.Tensor, h_anchor: torch.Tensor, L: int, B: int, T: int, d: int,
                  max_count: int) -> None:
    _need_cuda("y_anchor", y_anchor, (torch.float32,))
    _need_cuda("h_anchor", h_anchor, (torch.float32,))
    if tuple(y_anchor.shape) != (L, B, T, d):
        raise ValueError(f"y_anchor has shape {tuple(y_anchor.shape)}, expected {(L, B, T, d)}")
    if tuple(h_anchor.shape) != (L, B, max_count, T):
        raise ValueError(f"h_anchor has shape {tuple(h_anchor.shape)}, expected {(L, B, max_count, T)}")


def rm_sparse_ffn_stack(x: torch.Tensor, y: torch.Tensor, layers: Sequence[Layer], idx: torch.Tensor,
                        count: torch.Tensor, max_count: int, ws: torch.Tensor, eps: float = 1e-6, act: str = "silu",
                        stream=None) -> None:
    """L masked FFN layers in order; idx [L][B][d_ff], count [L][B]."""
    shape, arr, L, B, T = _stack_args(x, y, layers, idx, count, eps, act)
    wp, wn = _ws(ws)
    _check(load_library().rm_sparse_ffn_stack(ctypes.byref(shape), arr, L, B, T, x.data_ptr(), y.data_ptr(),
                                              idx.data_ptr(), count.data_ptr(), int(max_count), wp, wn,
                                              _stream(stream)))


def _masks(mask: torch.Tensor, idx: torch.Tensor, count: torch.Tensor, n: int, d_ff: int) -> None:
    _need_cuda("mask", mask, (torch.uint8, torch.bool))
    _need_cuda("idx", idx, (torch.int32,))
    _need_cuda("count", count, (torch.int32,))
    if mask.numel() != n * d_ff or idx.numel() != n * d_ff or count.numel() != n:
        raise ValueError(f"mask and idx must hold {n} x d_ff={d_ff} and count {n} entries")


def rm_masked_ffn_layer(x: torch.Tensor, y: torch.Tensor, layer: Layer, mask: torch.Tensor, idx: torch.Tensor,
                        count: torch.Tensor, max_count: int, ws: torch.Tensor, eps: float = 1e-6, act: str = "silu",
                        stream=None) -> None:
    """rm_mask_compact(mask -> idx, count) + rm_sparse_ffn_layer, the compaction inside the layer's first launch."""
    shape = _shape(layer, eps, act)
    B, T = _activations(x, y, shape.d)
    w = _weights(layer, B)
    _masks(mask, idx, count, B, shape.d_ff)
    wp, wn = _ws(ws)
    _check(load_library().rm_masked_ffn_layer(ctypes.byref(shape), ctypes.byref(w), B, T, x.data_ptr(),
                                              y.data_ptr(), mask.data_ptr(), idx.data_ptr(), count.data_ptr(),
                                              int(max_count), wp, wn, _stream(stream)))


def rm_masked_ffn_stack(x: torch.Tensor, y: torch.Tensor, layers: Sequence[Layer], mask: torch.Tensor,
                        idx: torch.Tensor, count: torch.Tensor, max_count: int, ws: torch.Tensor, eps: float = 1e-6,
                        act: str = "silu", stream=None) -> None:
    """rm_mask_compact of [L][B] masks + rm_sparse_ffn_stack, the compaction inside the stack's first launch."""
    shape, arr, L, B, T = _stack_args(x, y, layers, idx, count, eps, act)
    _masks(mask, idx, count, L * B, shape.d_ff)
    wp, wn = _ws(ws)
    _check(load_library().rm_masked_ffn_stack(ctypes.byref(shape), arr, L, B, T, x.data_ptr(), y.data_ptr(),
                                              mask.data_ptr(), idx.data_ptr(), count.data_ptr(), int(max_count),
                                              wp, wn, _stream(stream)))


def rm_anchor_ffn_stack(x: torch.Tensor, y: torch.Tensor, layers: Sequence[Layer], idx: torch.Tensor,
                        count: torch.Tensor, max_count: int, y_anchor: torch.Tensor, h_anchor: torch.Tensor,
                        ws: torch.Tensor, eps: float = 1e-6, act: str = "silu", stream=None) -> None:
    """Eq. 4 anchor step: L dense layers; keeps y_a [L][B][T][d] and h_a of the group's lists [L][B][max_count][T].
    The workspace is sized with max_count = d_ff."""
    shape, arr, L, B, T = _stack_args(x, y, layers, idx, count, eps, act)
    _anchor_state(y_anchor, h_anchor, L, B, T, shape.d, int(max_count))
    wp, wn = _ws(ws)
    _check(load_library().rm_anchor_ffn_stack(ctypes.byref(shape), arr, L, B, T, x.data_ptr(), y.data_ptr(),
                                              idx.data_ptr(), count.data_ptr(), int(max_count),
                                              y_anchor.data_ptr(), h_anchor.data_ptr(), wp, wn, _stream(stream)))


def rm_delta_ffn_stack(x: torch.Tensor, y: torch.Tensor, layers: Sequence[Layer], idx: torch.Tensor,
                       count: torch.Tensor, max_count: int, y_anchor: torch.Tensor, h_anchor: torch.Tensor,
                       ws: torch.Tensor, eps: float = 1e-6, act: str = "silu", stream=None) -> None:
    """Eq. 4 non-anchor step: y = x + y_a + (h - h_a) W_down over the listed neurons, per layer."""
    shape, arr, L, B, T = _stack_args(x, y, layers, idx, count, eps, act)
    _anchor_state(y_anchor, h_anchor, L, B, T, shape.d, int(max_count))
    wp, wn = _ws(ws)
    _check(load_library().rm_delta_ffn_stack(ctypes.byref(shape), arr, L, B, T, x.data_ptr(), y.data_ptr(),
                                             idx.data_ptr(), count.data_ptr(), int(max_count),
                                             y_anchor.data_ptr(), h_anchor.data_ptr(), wp, wn, _stream(stream)))


def rm_dense_ffn_ref(x: torch.Tensor, y: torch.Tensor, layer: Layer, ws: torch.Tensor, eps: float = 1e-6,
                     act: str = "silu", stream=None) -> None:
    """y = x + dense GLU FFN (every neuron)."""
    shape = _shape(layer, eps, act)
    B, T = _activations(x, y, shape.d)
    w = _weights(layer, B)
    wp, wn = _ws(ws)
    _check(load_library().rm_dense_ffn_ref(ctypes.byref(shape), ctypes.byref(w), B, T, x.data_ptr(), y.data_ptr(),
                                           wp, wn, _stream(stream)))


def rm_gather_stack_rows(layers: Sequence[Layer], idx: torch.Tensor, count: torch.Tensor, max_count: int,
                         out: torch.Tensor, stream=None) -> None:
    """Compact copies of each layer's listed rows: out [L][3][max_count][d] (w_gate, w_up, w_down rows), rows past
    a layer's count zero; idx [L][d_ff], count [L] (one list per layer)."""
    L = len(layers)
    if L == 0:
        raise ValueError("at least one layer")
    shape = _shape(layers[0], 1e-6)
    arr = (LayerWeights * L)()
    for l, layer in enumerate(layers):
        arr[l] = _weights(layer)
    _need_cuda("idx", idx, (torch.int32,))
    _need_cuda("count", count, (torch.int32,))
    _need_cuda("out", out, (layers[0][0].dtype,))
    if idx.numel() != L * shape.d_ff or count.numel() != L or out.numel() != L * 3 * max_count * shape.d:
        raise ValueError("idx must be [L][d_ff], count [L] and out [L][3][max_count][d]")
    _check(load_library().rm_gather_stack_rows(ctypes.byref(shape), arr, L, idx.data_ptr(), count.data_ptr(),
                                               int(max_count), out.data_ptr(), _stream(stream)))


def rm_context_select(x: torch.Tensor, x_ref: torch.Tensor, v0: int, P: int, k: int, drift: Optional[torch.Tensor],
                      rows: torch.Tensor, count: torch.Tensor, stream=None) -> None:
    """Eq. 2 drift of the visual rows [v0, v0 + P) of x [N][d] against x_ref, and the rows to recompute: every
    non-visual row plus the k visual rows of largest drift (ascending, in rows[:count[0]])."""
    _need_cuda("x", x, (torch.float32,), 2)
    _need_cuda("x_ref", x_ref, (torch.float32,), 2)
    if x.shape != x_ref.shape:
        raise ValueError("x and x_ref must have the same shape")
    n_tok, d = x.shape
    if drift is not None:
        _need_cuda("drift", drift, (torch.float32,))
        if drift.numel() < P:
            raise ValueError("drift must hold P entries")
    _need_cuda("rows", rows, (torch.int32,))
    _need_cuda("count", count, (torch.int32,))
    if rows.numel() < n_tok or count.numel() < 1:
        raise ValueError("rows must hold N entries and count one")
    _check(load_library().rm_context_select(x.data_ptr(), x_ref.data_ptr(), n_tok, d, int(v0), int(P), int(k),
                                            _ptr(drift), rows.data_ptr(), count.data_ptr(), _stream(stream)))


def context_workspace(d: int, d_ff: int, n_tok: int, max_rows: int, act: str = "gelu_tanh", device="cuda"):
    """A workspace tensor (uint8) of the size rm_context_workspace_size asks for."""
    out = ctypes.c_size_t(0)
    shape = FfnShape(d, d_ff, RM_BF16, 1e-6, ACTS[act])
    _check(load_library().rm_context_workspace_size(ctypes.byref(shape), n_tok, max_rows, ctypes.byref(out)))
    return torch.empty(int(out.value), dtype=torch.uint8, device=device)


def rm_context_ffn(x: torch.Tensor, y: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor,
                   w_down_t: torch.Tensor, rows: torch.Tensor, count: torch.Tensor, max_rows: int, ws: torch.Tensor,
                   act: str = "gelu_tanh", stream=None) -> None:
    """Eq. 3: y[rows[:count]] = F(x[rows[:count]]); other rows of y (the reference outputs) are left as they are.
    w_gate, w_up bf16 [d_ff][d]; w_down_t bf16 [d][d_ff] (nn.Linear layout)."""
    _need_cuda("x", x, (torch.float32,), 2)
    _need_cuda("y", y, (torch.float32,), 2)
    if x.shape != y.shape:
        raise ValueError("x and y must have the same shape")
    n_tok, d = x.shape
    _need_cuda("w_gate", w_gate, (torch.bfloat16,), 2)
    d_ff = w_gate.shape[0]
    for name, w, shp in (("w_gate", w_gate, (d_ff, d)), ("w_up", w_up, (d_ff, d)), ("w_down_t", w_down_t, (d, d_ff))):
        _need_cuda(name, w, (torch.bfloat16,), 2)
        if tuple(w.shape) != shp:
            raise ValueError(f"{name} has shape {tuple(w.shape)}, expected {shp}")
    _need_cuda("rows", rows, (torch.int32,))
    _need_cuda("count", count, (torch.int32,))
    if act not in ACTS:
        raise ValueError(f"act must be one of {sorted(ACTS)}")
    shape = FfnShape(d, d_ff, RM_BF16, 1e-6, ACTS[act])
    wp, wn = _ws(ws)
    _check(load_library().rm_context_ffn(ctypes.byref(shape), w_gate.data_ptr(), w_up.data_ptr(),
                                         w_down_t.data_ptr(), n_tok, x.data_ptr(), rows.data_ptr(), count.data_ptr(),
                                         int(max_rows), y.data_ptr(), wp, wn, _stream(stream)))


def rm_context_pack(w_gate: torch.Tensor, w_up: torch.Tensor, w_down_t: torch.Tensor, act: str = "gelu_tanh",
                    stream=None) -> torch.Tensor:
    """The layer's three matrices in the blocked layout rm_context_ffn_packed reads (a uint8 tensor of
    3 * d * d_ff * 2 bytes, allocated here).  Run once per layer when the weights are loaded."""
    _need_cuda("w_gate", w_gate, (torch.bfloat16,), 2)
    d_ff, d = w_gate.shape
    for name, w, shp in (("w_up", w_up, (d_ff, d)), ("w_down_t", w_down_t, (d, d_ff))):
        _need_cuda(name, w, (torch.bfloat16,), 2)
        if tuple(w.shape) != shp:
            raise ValueError(f"{name} has shape {tuple(w.shape)}, expected {shp}")
    if act not in ACTS:
        raise ValueError(f"act must be one of {sorted(ACTS)}")
    shape = FfnShape(d, d_ff, RM_BF16, 1e-6, ACTS[act])
    n = ctypes.c_size_t(0)
    lib = load_library()
    _check(lib.rm_context_pack_size(ctypes.byref(shape), ctypes.byref(n)))
    packed = torch.empty(int(n.value), dtype=torch.uint8, device=w_gate.device)
    _check(lib.rm_context_pack(ctypes.byref(shape), w_gate.data_ptr(), w_up.data_ptr(), w_down_t.data_ptr(),
                               packed.data_ptr(), packed.numel(), _stream(stream)))
    return packed


def rm_context_ffn_packed(x: torch.Tensor, y: torch.Tensor, packed: torch.Tensor, rows: torch.Tensor,
                          count: torch.Tensor, max_rows: int, ws: torch.Tensor, act: str = "gelu_tanh",
                          stream=None) -> None:
    """rm_context_ffn with the weights from rm_context_pack (d_ff follows from the packed size)."""
    _need_cuda("x", x, (torch.float32,), 2)
    _need_cuda("y", y, (torch.float32,), 2)
    if x.shape != y.shape:
        raise ValueError("x and y must have the same shape")
    n_tok, d = x.shape
    _need_cuda("packed", packed, (torch.uint8,))
    if packed.numel() % (6 * d) != 0:
        raise ValueError("packed does not hold the three matrices of a layer with this d")
    d_ff = packed.numel() // (6 * d)
    _need_cuda("rows", rows, (torch.int32,))
    _need_cuda("count", count, (torch.int32,))
    if act not in ACTS:
        raise ValueError(f"act must be one of {sorted(ACTS)}")
    shape = FfnShape(d, d_ff, RM_BF16, 1e-6, ACTS[act])
    wp, wn = _ws(ws)
    _check(load_library().rm_context_ffn_packed(ctypes.byref(shape), packed.data_ptr(), n_tok, x.data_ptr(),
                                                rows.data_ptr(), count.data_ptr(), int(max_rows), y.data_ptr(), wp,
                                                wn, _stream(stream)))


def rm_neuron_norms(w_down: torch.Tensor, norms: torch.Tensor, stream=None) -> None:
    """||W_down[n]||_2 per neuron (Eq. 1's weight factor): w_down [d_ff][d] -> norms float32 [d_ff]."""
    _need_cuda("w_down", w_down, (torch.float32, torch.bfloat16), 2)
    d_ff, d = w_down.shape
    _need_cuda("norms", norms, (torch.float32,))
    if norms.numel() != d_ff:
        raise ValueError(f"norms must hold d_ff={d_ff} entries")
    _check(load_library().rm_neuron_norms(w_down.data_ptr(), d_ff, d, wdtype_of(w_down), norms.data_ptr(),
                                          _stream(stream)))


def rm_group_masks(h: torch.Tensor, norms: torch.Tensor, k: int, scores: torch.Tensor, mask: torch.Tensor,
                   stream=None) -> None:
    """Group masks (section 5): h float32 [S][L][d_ff][T], norms [L][d_ff] -> scores float32 [S][L][d_ff] and
    mask uint8 [L][d_ff]."""
    _need_cuda("h", h, (torch.float32,), 4)
    S, L, d_ff, T = h.shape
    _need_cuda("norms", norms, (torch.float32,))
    _need_cuda("scores", scores, (torch.float32,))
    _need_cuda("mask", mask, (torch.uint8, torch.bool))
    if norms.numel() != L * d_ff or scores.numel() != S * L * d_ff or mask.numel() != L * d_ff:
        raise ValueError("norms must be [L][d_ff], scores [S][L][d_ff] and mask [L][d_ff]")
    _check(load_library().rm_group_masks(h.data_ptr(), S, L, d_ff, T, norms.data_ptr(), int(k), scores.data_ptr(),
                                         mask.data_ptr(), _stream(stream)))


_ATTN_DTYPES = {torch.float32: RM_F32, torch.bfloat16: RM_BF16}


class _Marshal(threading.local):
    """Per thread, the C structs of one call (the library reads them before it returns): up to 6 rm_heads and an
    rm_attn_shape, filled by one pack each, and their addresses."""

    def __init__(self):
        self.heads = ctypes.create_string_buffer(6 * ctypes.sizeof(Heads))
        self.shape = ctypes.create_string_buffer(ctypes.sizeof(AttnShape))
        base = ctypes.addressof(self.heads)
        self.at = [base + i * ctypes.sizeof(Heads) for i in range(6)]
        self.shape_at = ctypes.addressof(self.shape)


_marshal = _Marshal()
_pack_heads = [struct.Struct("=" + "Qqqq" * n).pack_into for n in range(7)]
_pack_shape = struct.Struct("=iiiiff").pack_into


def _heads4(name: str, t: torch.Tensor, dtype, index: int) -> Tuple[int, int, int, int]:
    """The fields of an rm_heads for a tensor of head vectors [B][T][H][D] on device `index`."""
    try:  # the usual case first
        b, n, h, c = t.stride()
        if c == 1 and t.dtype is dtype and t.get_device() == index:
            return t.data_ptr(), b, n, h
    except (AttributeError, ValueError):
        pass
    return _heads(name, t, dtype, index, 4)


def _heads3(name: str, t: torch.Tensor, dtype, index: int) -> Tuple[int, int, int, int]:
    """The same for [T][H][D]."""
    try:
        n, h, c = t.stride()
        if c == 1 and t.dtype is dtype and t.get_device() == index:
            return t.data_ptr(), 0, n, h
    except (AttributeError, ValueError):
        pass
    return _heads(name, t, dtype, index, 3)


def _heads(name: str, t: torch.Tensor, dtype, index: int, ndim: int) -> Tuple[int, int, int, int]:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.get_device() != index:
        raise ValueError(f"{name} must be on a HIP device, the same as the other tensors, got {t.device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got {tuple(t.shape)}")
    st = t.stride()
    if st[-1] != 1 and t.shape[-1] != 1:
        raise ValueError(f"{name}: the elements of a head must be consecutive")
    return t.data_ptr(), st[0] if ndim == 4 else 0, st[-3], st[-2]


def _vector(name: str, t: Optional[torch.Tensor], dtype, index: int, shape) -> Optional[int]:
    """Pointer of an optional contiguous tensor of a dtype, device and shape."""
    if t is None:
        return None
    try:  # the usual case first
        if t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _need_cuda(name, t, (dtype,))
    raise ValueError(f"{name} must be {dtype} {list(shape)} on device {index}, got {list(t.shape)} on {t.device}")


def _attn_device(t: torch.Tensor, stream) -> int:
    """The tensors' device, which has to be the current one (the kernels are launched there), as the stream's has."""
    try:
        index = t.get_device()
    except AttributeError:
        index = -1
    if index < 0:
        raise ValueError("tensors must be on a HIP device")
    if index != _current_device():
        raise ValueError(f"tensors are on {t.device}, which is not the current device")
    if stream is not None and getattr(stream, "device_index", index) != index:
        raise ValueError(f"the stream is of another device than the tensors, which are on {t.device}")
    return index


def _attn_shape(q: torch.Tensor, n_q_heads: int, n_kv_heads: int, D: int, scale: Optional[float],
                softcap: float) -> int:
    """Address of the call's rm_attn_shape."""
    dtype = _ATTN_DTYPES.get(q.dtype)
    if dtype is None:
        raise ValueError(f"queries must be float32 or bfloat16, got {q.dtype}")
    if scale is None:
        scale = D ** -0.5 if D > 0 else 1.0
    _pack_shape(_marshal.shape, 0, n_q_heads, n_kv_heads, D, dtype, scale, softcap)
    return _marshal.shape_at


def _attn_ws(ws: Optional[torch.Tensor], index: int) -> Tuple[Optional[int], int]:
    if ws is None:
        return None, 0
    if ws.dtype != torch.uint8 or ws.get_device() != index or not ws.is_contiguous():
        _need_cuda("ws", ws, (torch.uint8,))
        raise ValueError(f"ws must be on device {index}, got {ws.device}")
    return ws.data_ptr(), ws.numel()


def rm_qk_norm_rope(q: torch.Tensor, k: torch.Tensor, v: Optional[torch.Tensor], q_out: torch.Tensor,
                    k_out: torch.Tensor, v_out: Optional[torch.Tensor], pos: torch.Tensor,
                    inv_freq: Optional[torch.Tensor], gain_q: Optional[torch.Tensor] = None,
                    gain_k: Optional[torch.Tensor] = None, slot: Optional[torch.Tensor] = None, eps: float = 1e-6,
                    pairs: bool = False, stream=None) -> None:
    """q [N][Hq][D], k and v [N][Hk][D] (views of one projection's rows will do): queries normalized and rotated into
    q_out [N][Hq][D], keys into rows slot[n] (None: n) of k_out [rows][Hk][D], values copied into those of v_out."""
    dev = _attn_device(q, stream)
    src, dst = q.dtype, q_out.dtype
    if src not in _ATTN_DTYPES or dst not in _ATTN_DTYPES:
        raise ValueError("queries and outputs must be float32 or bfloat16")
    fields = (_heads3("q", q, src, dev) + _heads3("k", k, src, dev) + _heads3("q_out", q_out, dst, dev)
              + _heads3("k_out", k_out, dst, dev))
    shape, k_shape, ko_shape = q.shape, k.shape, k_out.shape
    N, Hq, D = shape
    Hk, rows = k_shape[1], ko_shape[0]
    if k_shape != (N, Hk, D) or q_out.shape != shape or ko_shape != (rows, Hk, D):
        raise ValueError("q and q_out must be [N][Hq][D], k [N][Hk][D] and k_out [rows][Hk][D]")
    if (v is None) != (v_out is None):
        raise ValueError("v and v_out go together")
    if v is not None:
        fields += _heads3("v", v, src, dev) + _heads3("v_out", v_out, dst, dev)
        if v.shape != k_shape or v_out.shape != ko_shape:
            raise ValueError("v must have k's shape and v_out k_out's")
    rot = 0 if inv_freq is None else 2 * inv_freq.shape[0]
    at = _marshal.at
    _pack_heads[len(fields) // 4](_marshal.heads, 0, *fields)
    _check(load_library().rm_qk_norm_rope(
        N, Hq, Hk, D, _ATTN_DTYPES[src], _ATTN_DTYPES[dst], at[0], at[1], None if v is None else at[4], at[2], at[3],
        None if v is None else at[5], rows, _vector("pos", pos, torch.int32, dev, (N,)),
        _vector("slot", slot, torch.int32, dev, (N,)), _vector("inv_freq", inv_freq, torch.float32, dev, (rot // 2,)),
        rot, pairs, _vector("gain_q", gain_q, torch.float32, dev, (D,)),
        _vector("gain_k", gain_k, torch.float32, dev, (D,)), eps, _stream(stream)))


def rm_attn_spans(span: torch.Tensor, N: int, causal: bool = True, window: int = 0,
                  q_start: Optional[torch.Tensor] = None, kv_len: Optional[torch.Tensor] = None,
                  prefix_len: Optional[torch.Tensor] = None, doc: Optional[torch.Tensor] = None, stream=None) -> None:
    """span int32 [B][T][2]: the interval of the N keys that each query row sees (see the header for the rules);
    q_start, kv_len, prefix_len int32 [B], doc int32 [B][N]."""
    dev = _attn_device(span, stream)
    B, T = span.shape[:2]
    i32 = torch.int32
    at = _vector("span", span, i32, dev, (B, T, 2))
    _check(load_library().rm_attn_spans(B, T, N, causal, window, _vector("q_start", q_start, i32, dev, (B,)),
                                        _vector("kv_len", kv_len, i32, dev, (B,)),
                                        _vector("prefix_len", prefix_len, i32, dev, (B,)),
                                        _vector("doc", doc, i32, dev, (B, N)), at, _stream(stream)))


def span_attention_workspace(q: torch.Tensor, k: torch.Tensor) -> torch.Tensor:
    """A workspace tensor (uint8) of the size rm_span_attention_workspace_size asks for (it may be 0)."""
    out = ctypes.c_size_t(0)
    shape = _attn_shape(q, q.shape[2], k.shape[2], q.shape[3], None, 0.0)
    _check(load_library().rm_span_attention_workspace_size(shape, q.shape[0], q.shape[1], k.shape[1],
                                                           ctypes.byref(out)))
    return torch.empty(int(out.value), dtype=torch.uint8, device=q.device)


def rm_span_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                      ws: Optional[torch.Tensor], span: Optional[torch.Tensor] = None,
                      slopes: Optional[torch.Tensor] = None, q_start: Optional[torch.Tensor] = None,
                      scale: Optional[float] = None, softcap: float = 0.0, stream=None) -> None:
    """out = softmax(cap(scale q k^T) - slopes |q_start + i - j|) v over each row's interval of keys (span None: all);
    scale None: 1 / sqrt(D)."""
    dev = _attn_device(q, stream)
    dtype = q.dtype
    fields = (_heads4("q", q, dtype, dev) + _heads4("k", k, dtype, dev) + _heads4("v", v, dtype, dev)
              + _heads4("out", out, dtype, dev))
    shape, k_shape = q.shape, k.shape
    B, T, Hq, D = shape
    N, Hk = k_shape[1], k_shape[2]
    if k_shape != (B, N, Hk, D) or v.shape != k_shape or out.shape != shape:
        raise ValueError("q and out must be [B][T][Hq][D], k and v [B][N][Hk][D]")
    wp, wn = _attn_ws(ws, dev)
    at = _marshal.at
    _pack_heads[4](_marshal.heads, 0, *fields)
    _check(load_library().rm_span_attention(
        _attn_shape(q, Hq, Hk, D, scale, softcap), B, T, N, at[0], at[1], at[2], at[3],
        _vector("span", span, torch.int32, dev, (B, T, 2)), _vector("slopes", slopes, torch.float32, dev, (Hq,)),
        _vector("q_start", q_start, torch.int32, dev, (B,)), wp, wn, _stream(stream)))


def prefix_attention_workspace(q: torch.Tensor, k_prefix: torch.Tensor, k_own: torch.Tensor) -> torch.Tensor:
    """A workspace tensor (uint8) of the size rm_prefix_attention_workspace_size asks for (it may be 0)."""
    out = ctypes.c_size_t(0)
    groups = k_prefix.shape[0]
    if groups <= 0 or q.shape[0] % groups != 0:
        raise ValueError("the samples must divide into the prefixes' groups")
    shape = _attn_shape(q, q.shape[2], k_own.shape[2], q.shape[3], None, 0.0)
    _check(load_library().rm_prefix_attention_workspace_size(shape, groups, q.shape[0] // groups, q.shape[1],
                                                             k_prefix.shape[1], k_own.shape[1], ctypes.byref(out)))
    return torch.empty(int(out.value), dtype=torch.uint8, device=q.device)


def rm_prefix_attention(q: torch.Tensor, k_prefix: torch.Tensor, v_prefix: torch.Tensor, k_own: torch.Tensor,
                        v_own: torch.Tensor, out: torch.Tensor, ws: Optional[torch.Tensor],
                        prefix_len: Optional[torch.Tensor] = None, own_len: Optional[torch.Tensor] = None,
                        causal: bool = False, scale: Optional[float] = None, softcap: float = 0.0, stream=None) -> None:
    """Samples q [groups * per_group][T][Hq][D] over their group's prefix keys k_prefix [groups][P][Hk][D] and their own
    k_own [groups * per_group][S][Hk][D], one softmax over both; scale None: 1 / sqrt(D)."""
    dev = _attn_device(q, stream)
    dtype = q.dtype
    fields = (_heads4("q", q, dtype, dev) + _heads4("k_prefix", k_prefix, dtype, dev)
              + _heads4("v_prefix", v_prefix, dtype, dev) + _heads4("k_own", k_own, dtype, dev)
              + _heads4("v_own", v_own, dtype, dev) + _heads4("out", out, dtype, dev))
    shape, p_shape, o_shape = q.shape, k_prefix.shape, k_own.shape
    B, T, Hq, D = shape
    groups, P, Hk, _ = p_shape
    S = o_shape[1]
    if groups <= 0 or B % groups != 0:
        raise ValueError("the samples must divide into the prefixes' groups")
    if (p_shape != (groups, P, Hk, D) or v_prefix.shape != p_shape or o_shape != (B, S, Hk, D)
            or v_own.shape != o_shape or out.shape != shape):
        raise ValueError("q and out must be [B][T][Hq][D], the prefix [groups][P][Hk][D], the own keys [B][S][Hk][D]")
    wp, wn = _attn_ws(ws, dev)
    at = _marshal.at
    _pack_heads[6](_marshal.heads, 0, *fields)
    _check(load_library().rm_prefix_attention(
        _attn_shape(q, Hq, Hk, D, scale, softcap), groups, B // groups, T, P, S, at[0], at[1], at[2],
        _vector("prefix_len", prefix_len, torch.int32, dev, (groups,)), at[3], at[4],
        _vector("own_len", own_len, torch.int32, dev, (B,)), causal, at[5], wp, wn, _stream(stream)))


def rm_page_slots(n_new: torch.Tensor, length: torch.Tensor, table: torch.Tensor, free_pages: torch.Tensor,
                  n_free: torch.Tensor, first: torch.Tensor, start: torch.Tensor, seq: torch.Tensor, pos: torch.Tensor,
                  slot: torch.Tensor, page: int, length_out: Optional[torch.Tensor] = None,
                  n_free_out: Optional[torch.Tensor] = None, refused: Optional[torch.Tensor] = None,
                  stream=None) -> None:
    """Appends n_new [B] tokens (negative: the request has ended) to requests of length [B] on pages of table
    [B][max_pages], pages taken from and given back to free_pages [n_pages], of which the first n_free [1] are free; the
    packed tokens' seq, pos and slot [max_tok], their requests' first [B + 1] and start [B].  length and n_free are updated
    in place unless length_out and n_free_out are given; all int32."""
    dev = _attn_device(table, stream)
    B, per = table.shape
    i32 = torch.int32
    n_tok, one = (seq.shape[0],), (1,)
    n_pages = free_pages.shape[0]
    at_len, at_free = _vector("length", length, i32, dev, (B,)), _vector("n_free", n_free, i32, dev, one)
    _check(load_library().rm_page_slots(
        B, seq.shape[0], page, n_pages, per, _vector("n_new", n_new, i32, dev, (B,)), at_len, at_free,
        _vector("table", table, i32, dev, (B, per)), _vector("free_pages", free_pages, i32, dev, (n_pages,)),
        at_len if length_out is None else _vector("length_out", length_out, i32, dev, (B,)),
        at_free if n_free_out is None else _vector("n_free_out", n_free_out, i32, dev, one),
        _vector("refused", refused, i32, dev, one), _vector("first", first, i32, dev, (B + 1,)),
        _vector("start", start, i32, dev, (B,)), _vector("seq", seq, i32, dev, n_tok),
        _vector("pos", pos, i32, dev, n_tok), _vector("slot", slot, i32, dev, n_tok), _stream(stream)))


def paged_attention_workspace(q: torch.Tensor, k_cache: torch.Tensor, table: torch.Tensor) -> torch.Tensor:
    """A workspace tensor (uint8) of the size rm_paged_attention_workspace_size asks for (it may be 0)."""
    out = ctypes.c_size_t(0)
    shape = _attn_shape(q, q.shape[1], k_cache.shape[2], q.shape[2], None, 0.0)
    _check(load_library().rm_paged_attention_workspace_size(shape, q.shape[0], k_cache.shape[1], table.shape[1],
                                                            ctypes.byref(out)))
    return torch.empty(int(out.value), dtype=torch.uint8, device=q.device)


def rm_paged_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor,
                       pos: torch.Tensor, out: torch.Tensor, ws: Optional[torch.Tensor],
                       seq: Optional[torch.Tensor] = None, window: int = 0, slopes: Optional[torch.Tensor] = None,
                       scale: Optional[float] = None, softcap: float = 0.0, stream=None) -> None:
    """Tokens q [N][Hq][D] at positions pos [N] of requests seq [N] (None: n) over their requests' keys up to pos in
    k_cache [n_pages][page][Hk][D] by table [n_seqs][max_pages]; scale None: 1 / sqrt(D)."""
    dev = _attn_device(q, stream)
    dtype = q.dtype
    fields = (_heads3("q", q, dtype, dev) + _heads4("k_cache", k_cache, dtype, dev)
              + _heads4("v_cache", v_cache, dtype, dev) + _heads3("out", out, dtype, dev))
    shape, k_shape = q.shape, k_cache.shape
    N, Hq, D = shape
    n_pages, page, Hk, _ = k_shape
    if k_shape[3] != D or v_cache.shape != k_shape or out.shape != shape:
        raise ValueError("q and out must be [N][Hq][D], k_cache and v_cache [n_pages][page][Hk][D]")
    n_seqs, per = table.shape
    wp, wn = _attn_ws(ws, dev)
    at = _marshal.at
    _pack_heads[4](_marshal.heads, 0, *fields)
    i32 = torch.int32
    _check(load_library().rm_paged_attention(
        _attn_shape(q, Hq, Hk, D, scale, softcap), N, n_seqs, page, n_pages, per, at[0], at[1], at[2], at[3],
        _vector("table", table, i32, dev, (n_seqs, per)), _vector("seq", seq, i32, dev, (N,)),
        _vector("pos", pos, i32, dev, (N,)), window, _vector("slopes", slopes, torch.float32, dev, (Hq,)), wp, wn,
        _stream(stream)))


def _modulation(name: str, t: torch.Tensor, index: int, shape) -> Tuple[int, int]:
    """Pointer and row stride of a float32 [B][d] tensor whose rows are contiguous."""
    try:
        row, c = t.stride()
        if c == 1 and t.dtype is torch.float32 and t.shape == shape and t.get_device() == index:
            return t.data_ptr(), row
    except (AttributeError, ValueError):
        pass
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    raise ValueError(f"{name} must be float32 {list(shape)} on device {index} with contiguous rows, got {t.dtype} "
                     f"{list(t.shape)} on {t.device}")


def rm_block_norm(x: torch.Tensor, f: Optional[torch.Tensor], y: Optional[torch.Tensor], out: Optional[torch.Tensor],
                  norm_post: bool = False, gain_post: Optional[torch.Tensor] = None,
                  gate: Optional[torch.Tensor] = None, gain_pre: Optional[torch.Tensor] = None,
                  scale: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None, x_scale: float = 1.0,
                  f_scale: float = 1.0, eps: float = 1e-6, stream=None) -> None:
    """y = x_scale x + f_scale gate norm_post(f), out = norm(y) gain_pre (1 + scale) + shift, all [B][T][d]; gains float32
    [d], gate, scale and shift float32 [B][d] (rows any multiple of 4 elements apart).  y may be x, out may be f."""
    dev = _attn_device(x, stream)
    shape = x.shape
    if len(shape) != 3:
        raise ValueError(f"x must be [B][T][d], got {list(shape)}")
    B, T, d = shape
    xt = x.dtype
    ft = xt if f is None else f.dtype
    ot = xt if out is None else out.dtype
    try:
        xd, fd, od = _ATTN_DTYPES[xt], _ATTN_DTYPES[ft], _ATTN_DTYPES[ot]
    except KeyError:
        raise ValueError("x, f and out must be float32 or bfloat16") from None
    f32 = torch.float32
    gp = sp = hp = g1 = g2 = None
    gs = ss = hs = 0
    if gate is not None:
        gp, gs = _modulation("gate", gate, dev, (B, d))
    if scale is not None:
        sp, ss = _modulation("scale", scale, dev, (B, d))
    if shift is not None:
        hp, hs = _modulation("shift", shift, dev, (B, d))
    if gain_post is not None:
        g1 = _vector("gain_post", gain_post, f32, dev, (d,))
    if gain_pre is not None:
        g2 = _vector("gain_pre", gain_pre, f32, dev, (d,))
    _check(load_library().rm_block_norm(
        B, T, d, xd, fd, od, _vector("x", x, xt, dev, shape), _vector("f", f, ft, dev, shape), norm_post, g1, gp, gs, x_scale,
        f_scale, _vector("y", y, xt, dev, shape), g2, sp, ss, hp, hs, eps, _vector("out", out, ot, dev, shape),
        _stream(stream)))


def rm_profile_kernel_events(kernel: int, ev_begin: Optional[int], ev_end: Optional[int]) -> None:
    """Arm raw hipEvent_t handles around the next launch of `kernel` (an RM_KERNEL_* id)."""
    _check(load_library().rm_profile_kernel_events(kernel, ev_begin, ev_end))


def rm_stream_read(buf: torch.Tensor, workgroups: int, sink: torch.Tensor, stream=None) -> None:
    """Measurement: a plain streaming read of the whole of `buf` (any dtype, 16-byte multiple); sink int32/uint8
    scratch of at least workgroups * 512 * 4 bytes."""
    if buf.device.type != "cuda" or not buf.is_contiguous():
        raise ValueError("buf must be a contiguous device tensor")
    _need_cuda("sink", sink, (torch.int32, torch.uint8))
    if sink.numel() * sink.element_size() < workgroups * 512 * 4:
        raise ValueError("sink must hold workgroups * 512 uint32")
    _check(load_library().rm_stream_read(buf.data_ptr(), buf.numel() * buf.element_size(), int(workgroups),
                                         sink.data_ptr(), _stream(stream)))

"""ctypes binding of liblasnet's C ABI (include/lasnet.h): argument marshalling only.

Every step of the path runs in the library's HIP kernels; PyTorch supplies device memory
and the current stream.  There is no fallback: a missing library or a failing call raises.
"""
from __future__ import annotations

import ctypes
import os
import warnings
from typing import Optional, Tuple

import torch

# LASNET_LIBRARY overrides the in-tree library (e.g. an instrumented build of the same sources).
_LIB_PATH = os.environ.get("LASNET_LIBRARY") or os.path.join(
    os.path.dirname(os.path.abspath(__file__)), "liblasnet.so")
_lib = None
_marshal = None

LASNET_F32, LASNET_BF16, LASNET_E4M3, LASNET_E8M0 = 0, 1, 2, 3
LASNET_POST_RELU, LASNET_FORCE_GENERIC, LASNET_SKIP_IDENTITY, LASNET_FORCE_FUSED, LASNET_FORCE_TILED = 1, 2, 4, 8, 16
LASNET_WEIGHTS_OF_ALL = 32
LASNET_OK, LASNET_EINVAL, LASNET_ESHAPE, LASNET_EUNSUPPORTED, LASNET_EALIAS, LASNET_EHIP = 0, -1, -2, -3, -4, -5
LASNET_ETOOBIG = -6
LASNET_NOALLOC_MAX_PACKED_BYTES = 4 << 20

EXPORTS = (
    "lasnet_version", "lasnet_status_string", "lasnet_masker", "lasnet_masker_ex", "lasnet_masker_logits",
    "lasnet_sparse_bottleneck", "lasnet_sparse_bottleneck_ex", "lasnet_dense_bottleneck",
    "lasnet_has_fast_path", "lasnet_packed_weights_bytes", "lasnet_pack_weights",
    "lasnet_sparse_bottleneck_packed", "lasnet_sparse_bottleneck_noalloc",
    "lasnet_workspace_bytes", "lasnet_sparse_bottleneck_planned",
    "lasnet_microbench_mfma", "lasnet_microbench_copy", "lasnet_microbench_weight_stream",
    "lasnet_norm_rows", "lasnet_norm_rows_backward", "lasnet_norm_rows_backward_workspace_bytes",
    "lasnet_route", "lasnet_route_workspace_bytes", "lasnet_dispatch_rows", "lasnet_combine_rows",
    "lasnet_combine_rows_backward", "lasnet_expert_product", "lasnet_expert_product_dx", "lasnet_expert_product_dw",
    "lasnet_expert_product_dw_ex", "lasnet_expert_product_dw_workspace_bytes",
    "lasnet_choose_experts", "lasnet_choose_experts_backward", "lasnet_balance", "lasnet_balance_workspace_bytes",
    "lasnet_quantize_rows", "lasnet_quantize_matrices", "lasnet_block_product",
)


# the calls on rows that _marshal takes
_ROW_CALLS = ("norm_rows", "norm_rows_backward", "route", "dispatch_rows", "combine_rows", "combine_rows_backward", "expert_product",
              "expert_product_dx", "expert_product_dw_ex", "choose_experts", "choose_experts_backward", "balance", "quantize_rows", "quantize_matrices",
              "block_product")


class LasnetError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().lasnet_status_string(status).decode()
        super().__init__("%s failed: %s (status %d)" % (where, msg, status))


class lasnet_tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_int32), ("h", ctypes.c_int32),
                ("w", ctypes.c_int32), ("c", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class lasnet_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("stride", ctypes.c_int64),
                ("cols", ctypes.c_int32), ("dtype", ctypes.c_int32)]


def load_library(path: str) -> ctypes.CDLL:
    """Loads one build of the library and declares the argument types of its entry points."""
    if not os.path.exists(path):
        raise RuntimeError(
            "liblasnet.so is not built (%s missing): run `python -m paper_2210_06223_amd.build`; "
            "there is no CPU fallback" % path)
    _load_marshal()
    L = ctypes.CDLL(path)
    vp, ip, tp = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(lasnet_tensor)
    L.lasnet_version.restype = ip
    L.lasnet_version.argtypes = []
    L.lasnet_status_string.restype = ctypes.c_char_p
    L.lasnet_status_string.argtypes = [ip]
    L.lasnet_masker.restype = ip
    L.lasnet_masker.argtypes = [tp, vp, ctypes.c_float, ip, ctypes.c_float, vp, vp, vp, vp]
    L.lasnet_masker_ex.restype = ip
    L.lasnet_masker_ex.argtypes = [tp, vp, ctypes.c_float, ip, ctypes.c_float, vp, vp, vp, tp, vp]
    L.lasnet_masker_logits.restype = ip
    L.lasnet_masker_logits.argtypes = [tp, vp, ctypes.c_float, ip, vp, vp]
    L.lasnet_sparse_bottleneck.restype = ip
    L.lasnet_sparse_bottleneck.argtypes = [tp, vp, vp, ip, ip, vp, vp, vp, vp, vp, vp, tp, vp]
    L.lasnet_sparse_bottleneck_ex.restype = ip
    L.lasnet_sparse_bottleneck_ex.argtypes = [tp, vp, vp, ip, ip, vp, vp, vp, vp, vp, vp, tp,
                                              ctypes.c_uint32, vp]
    L.lasnet_workspace_bytes.restype = ctypes.c_size_t
    L.lasnet_workspace_bytes.argtypes = [ip] * 7
    L.lasnet_sparse_bottleneck_planned.restype = ip
    L.lasnet_sparse_bottleneck_planned.argtypes = [tp, vp, vp, vp, ip, ip, vp, vp, vp, vp, tp, ctypes.c_uint32,
                                                   vp, ctypes.c_size_t, vp]
    L.lasnet_microbench_mfma.restype = ctypes.c_double
    L.lasnet_microbench_mfma.argtypes = [ip, vp, vp]
    L.lasnet_microbench_weight_stream.restype = ctypes.c_double
    L.lasnet_microbench_weight_stream.argtypes = [vp, ctypes.c_size_t, ip, vp, vp]
    L.lasnet_microbench_copy.restype = ip
    L.lasnet_microbench_copy.argtypes = [vp, vp, ctypes.c_size_t, vp]
    L.lasnet_sparse_bottleneck_noalloc.restype = ip
    L.lasnet_sparse_bottleneck_noalloc.argtypes = L.lasnet_sparse_bottleneck_ex.argtypes
    L.lasnet_dense_bottleneck.restype = ip
    L.lasnet_dense_bottleneck.argtypes = [tp, ip, vp, vp, vp, vp, vp, vp, tp, ctypes.c_uint32, vp]
    L.lasnet_has_fast_path.restype = ip
    L.lasnet_has_fast_path.argtypes = [ip, ip, ip, ip]
    L.lasnet_packed_weights_bytes.restype = ctypes.c_size_t
    L.lasnet_packed_weights_bytes.argtypes = [ip, ip, ip, ip]
    L.lasnet_pack_weights.restype = ip
    L.lasnet_pack_weights.argtypes = [ip, ip, ip, ip, vp, vp, vp, vp, vp]
    L.lasnet_sparse_bottleneck_packed.restype = ip
    L.lasnet_sparse_bottleneck_packed.argtypes = [tp, vp, vp, ip, ip, vp, vp, vp, vp, tp,
                                                  ctypes.c_uint32, vp]
    rp, sz, i64 = ctypes.POINTER(lasnet_rows), ctypes.c_size_t, ctypes.c_int64
    for name, result, args in (
            ("norm_rows", ip, [rp, rp, vp, ctypes.c_float, rp, rp, vp, vp, vp]),
            ("norm_rows_backward_workspace_bytes", sz, [i64, ip]),
            ("norm_rows_backward", ip, [rp, rp, vp, vp, rp, rp, vp, vp, sz, vp]),
            ("route_workspace_bytes", sz, [i64, ip, ip]),
            ("route", ip, [vp, i64, ip, ip, vp, vp, vp, vp, sz, vp]),
            ("dispatch_rows", ip, [rp, vp, vp, vp, ip, ip, rp, vp, vp]),
            ("combine_rows", ip, [rp, vp, vp, ip, rp, rp, vp]),
            ("combine_rows_backward", ip, [rp, rp, vp, vp, vp, ip, ip, rp, vp, vp]),
            ("expert_product", ip, [rp, vp, vp, ip, vp, vp, rp, ctypes.c_uint32, vp]),
            ("expert_product_dx", ip, [rp, vp, ip, vp, rp, vp]),
            ("expert_product_dw", ip, [rp, rp, vp, ip, vp, ip, vp]),
            ("expert_product_dw_workspace_bytes", sz, [i64, ip, ip, ip]),
            ("expert_product_dw_ex", ip, [rp, rp, vp, ip, vp, ip, vp, sz, vp]),
            ("choose_experts", ip, [rp, vp, ip, vp, vp, vp, ctypes.c_uint32, vp]),
            ("choose_experts_backward", ip, [rp, vp, vp, vp, ip, vp, vp, vp, rp, ctypes.c_uint32, vp]),
            ("balance_workspace_bytes", sz, [i64, ip]),
            ("balance", ip, [rp, vp, vp, ip, vp, vp, vp, vp, sz, vp]),
            ("quantize_rows", ip, [rp, vp, vp, ip, ip, rp, vp, vp]),
            ("quantize_matrices", ip, [vp, ip, ip, ip, ip, vp, vp, vp, vp, vp]),
            ("block_product", ip, [rp, vp, vp, ip, vp, vp, ip, rp, ctypes.c_uint32, vp])):
        f = getattr(L, "lasnet_" + name)
        f.restype, f.argtypes = result, args
    # the entry points that _marshal calls, by address
    L.at_masker_ex, L.at_ex, L.at_dense, L.at_packed, L.at_planned, L.at_packed_bytes = (
        ctypes.cast(f, vp).value for f in (L.lasnet_masker_ex, L.lasnet_sparse_bottleneck_ex, L.lasnet_dense_bottleneck,
                                           L.lasnet_sparse_bottleneck_packed, L.lasnet_sparse_bottleneck_planned,
                                           L.lasnet_packed_weights_bytes))
    for name in _ROW_CALLS:
        setattr(L, "at_" + name, ctypes.cast(getattr(L, "lasnet_" + name), vp).value)
    return L


class _AllThroughCtypes:
    """In place of the native marshalling where it does not load: no call is of its form."""
    masker_ex = block_ex = block_dense = block_packed = block_planned = staticmethod(lambda *args: None)
    norm_rows = norm_rows_backward = route = dispatch_rows = combine_rows = combine_rows_backward = masker_ex
    expert_product = expert_product_dx = expert_product_dw = masker_ex
    choose_experts = choose_experts_backward = balance = quantize_rows = quantize_matrices = block_product = masker_ex


def _load_marshal() -> None:
    """The extension saves host time and nothing else: the ctypes calls below are complete without it."""
    global _marshal
    if _marshal is None:
        try:
            from . import _marshal as m
        except ImportError as e:                 # not built, or built against another torch
            warnings.warn("the native marshalling does not load (%s); calls take some 5 us longer on the host until "
                          "`python -m paper_2210_06223_amd.build` has made it anew" % e, RuntimeWarning, stacklevel=3)
            m = _AllThroughCtypes
        _marshal = m


def lib() -> ctypes.CDLL:
    """The in-tree liblasnet.so (built by paper_2210_06223_amd.build / __graft_entry__.build)."""
    global _lib
    if _lib is None:
        _lib = load_library(_LIB_PATH)
    return _lib


# Host time per call matters at a few images, where a block's kernels take 20 us.  A call on the current stream that brings all of its
# outputs is offered to the native marshalling (csrc/marshal.cpp), which takes it if its arguments are of the plain form (tensors as the
# checks below ask for) and answers None for any other; that, and a call that is not offered, goes through the checks, conversions and ctypes call below.  There addresses go to
# ctypes as plain integers (argtypes makes them pointers), and the current stream's handle is read without building a
# torch.cuda.Stream object (3.0 -> 0.2 us).  masker_ex + packed block, one
# 14x14x1024 image: 25.4 us without any of it, 24.2 with ctypes and integers, 16.3 marshalled natively, of which the five launches
# take 16.
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


_DTYPES = {torch.float32: LASNET_F32, torch.bfloat16: LASNET_BF16}


def _as_tensor_desc(x: torch.Tensor) -> lasnet_tensor:
    shape = x.shape
    if len(shape) != 4 or not x.is_contiguous():
        raise ValueError("feature maps are contiguous NHWC tensors [N,H,W,C]")
    dt = _DTYPES.get(x.dtype)
    if dt is None:
        raise ValueError("dtype must be float32 or bfloat16")
    if not x.is_cuda:
        raise ValueError("feature maps live in device memory")
    return lasnet_tensor(x.data_ptr() or None, *shape, dt)


def _empty(shape, dtype: torch.dtype, device, stream, output: bool = False) -> torch.Tensor:
    """What a call makes is memory of the stream that the call runs on: a block of the current stream's pool may have a last user there that has not finished,
    and the call's kernels would not wait for it.  An output will be used on the caller's current stream, too: freed, it is not given away before that has come so far.
    (A stream of another kind is known by its handle.  An output on another stream takes the host 7 us more, by torch.cuda.stream(), which does the same, 12.)"""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    here, gpu = torch.cuda.current_stream(device), torch._C._cuda_getDevice()
    if stream == here:
        return torch.empty(shape, dtype=dtype, device=device)
    _switch(stream)
    try:
        t = torch.empty(shape, dtype=dtype, device=device)
    finally:
        _switch(here)
        if here.device_index != gpu:
            torch._C._cuda_setDevice(gpu)
    if output:
        t.record_stream(here)
    return t


def _switch(stream) -> None:
    torch._C._cuda_setStream(stream_id=stream.stream_id, device_index=stream.device_index, device_type=stream.device_type)


def _output(shape, dtype: torch.dtype, device, stream) -> torch.Tensor:
    return _empty(shape, dtype, device, stream, True)


def _check(status: int, where: str):
    if status != LASNET_OK:
        raise LasnetError(status, where)


def _f32(t: torch.Tensor, name: str) -> torch.Tensor:
    if t.dtype != torch.float32 or not t.is_contiguous() or not t.is_cuda:
        raise ValueError("%s must be a contiguous float32 device tensor" % name)
    return t


def lasnet_version() -> int:
    return lib().lasnet_version()


def lasnet_has_fast_path(dtype: torch.dtype, C: int, M: int, S: int) -> int:
    return lib().lasnet_has_fast_path(LASNET_BF16 if dtype == torch.bfloat16 else LASNET_F32, C, M, S)


def lasnet_masker(x: torch.Tensor, Wm: torch.Tensor, bm: float, S: int, thr: float = 0.0,
                  mask: Optional[torch.Tensor] = None, idx: Optional[torch.Tensor] = None,
                  count: Optional[torch.Tensor] = None, stream=None
                  ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """mask uint8 [N,G,GW], idx int32 [N*G*GW] (first count valid), count int32 [1]; all on device."""
    if stream is None and mask is not None and idx is not None and count is not None:
        L = lib()
        st = _marshal.masker_ex(L.at_masker_ex, x, Wm, bm, S, thr, mask, idx, count, None)
        if st is not None:
            _check(st, "lasnet_masker")
            return mask, idx, count
    d = _as_tensor_desc(x)
    N, H, W, _ = x.shape
    if S <= 0 or H % S or W % S:
        _check(LASNET_ESHAPE if S > 0 else LASNET_EINVAL, "lasnet_masker")
    G, GW = H // S, W // S
    if mask is None:
        mask = _output((N, G, GW), torch.uint8, x.device, stream)
    if idx is None:
        idx = _output((N * G * GW,), torch.int32, x.device, stream)
    if count is None:
        count = _output((1,), torch.int32, x.device, stream)
    st = lib().lasnet_masker(ctypes.byref(d), _ptr(_f32(Wm, "Wm")), float(bm), int(S), float(thr),
                             _ptr(mask), _ptr(idx), _ptr(count), _stream(stream))
    _check(st, "lasnet_masker")
    return mask, idx, count


def lasnet_masker_ex(x: torch.Tensor, Wm: torch.Tensor, bm: float, S: int, thr: float = 0.0,
                     mask: Optional[torch.Tensor] = None, idx: Optional[torch.Tensor] = None,
                     count: Optional[torch.Tensor] = None, pass_out: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """lasnet_masker that also copies every inactive cell of x to pass_out (may be None)."""
    if stream is None and mask is not None and idx is not None and count is not None:
        L = lib()
        st = _marshal.masker_ex(L.at_masker_ex, x, Wm, bm, S, thr, mask, idx, count, pass_out)
        if st is not None:
            _check(st, "lasnet_masker_ex")
            return mask, idx, count
    d = _as_tensor_desc(x)
    N, H, W, _ = x.shape
    if S <= 0 or H % S or W % S:
        _check(LASNET_ESHAPE if S > 0 else LASNET_EINVAL, "lasnet_masker_ex")
    G, GW = H // S, W // S
    if mask is None:
        mask = _output((N, G, GW), torch.uint8, x.device, stream)
    if idx is None:
        idx = _output((N * G * GW,), torch.int32, x.device, stream)
    if count is None:
        count = _output((1,), torch.int32, x.device, stream)
    po = None
    if pass_out is not None:
        po = _as_tensor_desc(pass_out)
    st = lib().lasnet_masker_ex(ctypes.byref(d), _ptr(_f32(Wm, "Wm")), float(bm), int(S), float(thr),
                                _ptr(mask), _ptr(idx), _ptr(count),
                                ctypes.byref(po) if po is not None else None, _stream(stream))
    _check(st, "lasnet_masker_ex")
    return mask, idx, count


def lasnet_masker_logits(x: torch.Tensor, Wm: torch.Tensor, bm: float, S: int,
                         logits: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    d = _as_tensor_desc(x)
    N, H, W, _ = x.shape
    if S <= 0 or H % S or W % S:
        _check(LASNET_ESHAPE if S > 0 else LASNET_EINVAL, "lasnet_masker_logits")
    if logits is None:
        logits = _output((N, H // S, W // S), torch.float64, x.device, stream)
    st = lib().lasnet_masker_logits(ctypes.byref(d), _ptr(_f32(Wm, "Wm")), float(bm), int(S),
                                    _ptr(logits), _stream(stream))
    _check(st, "lasnet_masker_logits")
    return logits


def _weights(x, W1, b1, W2, b2, W3, b3):
    for n, t in (("W1", W1), ("W2", W2), ("W3", W3)):
        if t.dtype != x.dtype or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("%s must be a contiguous device tensor of x's dtype" % n)
    M, C = W1.shape
    if C != x.shape[3] or tuple(W2.shape) != (M, 3, 3, M) or tuple(W3.shape) != (C, M):
        raise ValueError("weights: W1 [M,C], W2 [M,3,3,M], W3 [C,M]")
    if b1.numel() != M or b2.numel() != M or b3.numel() != C:
        raise ValueError("biases: b1 [M], b2 [M], b3 [C]")
    return int(M), [_ptr(W1), _ptr(_f32(b1, "b1")), _ptr(W2), _ptr(_f32(b2, "b2")), _ptr(W3),
                    _ptr(_f32(b3, "b3"))]


def _check_list(d: lasnet_tensor, idx: Optional[torch.Tensor], count: Optional[torch.Tensor], S: int) -> None:
    """The list's storage is what the masker writes to: room for every cell of the map (the kernels may read
    entries past count[0], which only the device knows; they never use them)."""
    if count is not None and (count.dtype != torch.int32 or not count.is_cuda or not count.is_contiguous()):
        raise ValueError("count must be a contiguous int32 device tensor")
    if idx is not None:
        if idx.dtype != torch.int32 or not idx.is_cuda or not idx.is_contiguous():
            raise ValueError("idx must be a contiguous int32 device tensor")
        if S > 0 and d.h % S == 0 and d.w % S == 0:
            cells = d.n * (d.h // S) * (d.w // S)
            if idx.numel() < cells:
                raise ValueError("idx must have room for all %d cells of the map (it holds %d entries)" % (cells, idx.numel()))


def lasnet_sparse_bottleneck(x: torch.Tensor, idx: Optional[torch.Tensor],
                             count: Optional[torch.Tensor], S: int, W1, b1, W2, b2, W3, b3,
                             out: Optional[torch.Tensor] = None, flags: int = 0,
                             stream=None) -> torch.Tensor:
    if stream is None and out is not None:
        L = lib()
        st = _marshal.block_ex(L.at_ex, x, idx, count, S, W1, b1, W2, b2, W3, b3, out, flags)
        if st is not None:
            _check(st, "lasnet_sparse_bottleneck")
            return out
    d = _as_tensor_desc(x)
    if out is None:
        out = _output(x.shape, x.dtype, x.device, stream)
    o = _as_tensor_desc(out)
    M, w = _weights(x, W1, b1, W2, b2, W3, b3)
    _check_list(d, idx, count, int(S))
    if flags:
        st = lib().lasnet_sparse_bottleneck_ex(ctypes.byref(d), _ptr(idx), _ptr(count), int(S), M, *w,
                                               ctypes.byref(o), int(flags), _stream(stream))
    else:
        st = lib().lasnet_sparse_bottleneck(ctypes.byref(d), _ptr(idx), _ptr(count), int(S), M, *w,
                                            ctypes.byref(o), _stream(stream))
    _check(st, "lasnet_sparse_bottleneck")
    return out


def lasnet_workspace_bytes(x: torch.Tensor, M: int, S: int) -> int:
    """Device memory the tiled schedule needs for a call on x (0: the fused schedule runs, or no fast path)."""
    n, h, w, c = x.shape
    return int(lib().lasnet_workspace_bytes(LASNET_BF16 if x.dtype == torch.bfloat16 else LASNET_F32,
                                            int(n), int(h), int(w), int(c), int(M), int(S)))


def lasnet_sparse_bottleneck_planned(x: torch.Tensor, idx: Optional[torch.Tensor],
                                     count: Optional[torch.Tensor], mask: Optional[torch.Tensor], S: int, M: int,
                                     packed: torch.Tensor, b1, b2, b3, out: torch.Tensor,
                                     workspace: Optional[torch.Tensor], flags: int = 0, stream=None) -> torch.Tensor:
    """The explicit form: packed weights, workspace (a uint8 device tensor or None) and out are the caller's."""
    if stream is None:
        L = lib()
        st = _marshal.block_planned(L.at_planned, x, idx, count, mask, S, M, packed, b1, b2, b3, out, workspace, flags)
        if st is not None:
            _check(st, "lasnet_sparse_bottleneck_planned")
            return out
    d = _as_tensor_desc(x)
    o = _as_tensor_desc(out)
    _check_list(d, idx, count, int(S))
    if mask is not None and (mask.dtype != torch.uint8 or not mask.is_cuda or not mask.is_contiguous()):
        raise ValueError("mask must be a contiguous uint8 device tensor")
    if b1.numel() != M or b2.numel() != M or b3.numel() != x.shape[3]:
        raise ValueError("biases: b1 [M], b2 [M], b3 [C]")
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = lib().lasnet_sparse_bottleneck_planned(ctypes.byref(d), _ptr(idx), _ptr(count), _ptr(mask), int(S), int(M),
                                                _ptr(packed), _ptr(_f32(b1, "b1")), _ptr(_f32(b2, "b2")),
                                                _ptr(_f32(b3, "b3")), ctypes.byref(o), int(flags),
                                                _ptr(workspace), wbytes, _stream(stream))
    _check(st, "lasnet_sparse_bottleneck_planned")
    return out


def lasnet_sparse_bottleneck_noalloc(x: torch.Tensor, idx: Optional[torch.Tensor],
                                     count: Optional[torch.Tensor], S: int, W1, b1, W2, b2, W3, b3,
                                     out: torch.Tensor, flags: int = 0, stream=None) -> torch.Tensor:
    """lasnet_sparse_bottleneck_ex whose weight repack goes to the library's fixed scratch array; `out` is
    the caller's (this wrapper allocates nothing either)."""
    d = _as_tensor_desc(x)
    o = _as_tensor_desc(out)
    M, w = _weights(x, W1, b1, W2, b2, W3, b3)
    _check_list(d, idx, count, int(S))
    st = lib().lasnet_sparse_bottleneck_noalloc(ctypes.byref(d), _ptr(idx), _ptr(count), int(S), M, *w,
                                                ctypes.byref(o), int(flags), _stream(stream))
    _check(st, "lasnet_sparse_bottleneck_noalloc")
    return out


def lasnet_dense_bottleneck(x: torch.Tensor, W1, b1, W2, b2, W3, b3,
                            out: Optional[torch.Tensor] = None, flags: int = 0,
                            stream=None) -> torch.Tensor:
    if stream is None and out is not None:
        L = lib()
        st = _marshal.block_dense(L.at_dense, x, W1, b1, W2, b2, W3, b3, out, flags)
        if st is not None:
            _check(st, "lasnet_dense_bottleneck")
            return out
    d = _as_tensor_desc(x)
    if out is None:
        out = _output(x.shape, x.dtype, x.device, stream)
    o = _as_tensor_desc(out)
    M, w = _weights(x, W1, b1, W2, b2, W3, b3)
    st = lib().lasnet_dense_bottleneck(ctypes.byref(d), M, *w, ctypes.byref(o), int(flags),
                                       _stream(stream))
    _check(st, "lasnet_dense_bottleneck")
    return out


def lasnet_pack_weights(S: int, W1: torch.Tensor, W2: torch.Tensor, W3: torch.Tensor,
                        packed: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Repack W1 [M,C], W2 [M,3,3,M], W3 [C,M] (bf16) for the matrix-core kernel of (C, M, S)."""
    M, C = W1.shape
    for n, t in (("W1", W1), ("W2", W2), ("W3", W3)):
        if t.dtype != torch.bfloat16 or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("%s must be a contiguous bfloat16 device tensor" % n)
    if tuple(W2.shape) != (M, 3, 3, M) or tuple(W3.shape) != (C, M):
        raise ValueError("weights: W1 [M,C], W2 [M,3,3,M], W3 [C,M]")
    nbytes = lib().lasnet_packed_weights_bytes(LASNET_BF16, int(C), int(M), int(S))
    if nbytes == 0:
        _check(LASNET_EUNSUPPORTED, "lasnet_pack_weights")
    if packed is None:
        packed = _output((nbytes // 2,), torch.bfloat16, W1.device, stream)
    elif packed.numel() * packed.element_size() < nbytes or not packed.is_cuda:
        raise ValueError("packed buffer too small")
    st = lib().lasnet_pack_weights(LASNET_BF16, int(C), int(M), int(S), _ptr(W1), _ptr(W2), _ptr(W3),
                                   _ptr(packed), _stream(stream))
    _check(st, "lasnet_pack_weights")
    return packed


def lasnet_sparse_bottleneck_packed(x: torch.Tensor, idx: Optional[torch.Tensor],
                                    count: Optional[torch.Tensor], S: int, M: int,
                                    packed: torch.Tensor, b1, b2, b3,
                                    out: Optional[torch.Tensor] = None, flags: int = 0,
                                    stream=None) -> torch.Tensor:
    if stream is None and out is not None:
        L = lib()
        st = _marshal.block_packed(L.at_packed, x, idx, count, S, M, packed, L.at_packed_bytes, b1, b2, b3, out, flags)
        if st is not None:
            _check(st, "lasnet_sparse_bottleneck_packed")
            return out
    d = _as_tensor_desc(x)
    if out is None:
        out = _output(x.shape, x.dtype, x.device, stream)
    o = _as_tensor_desc(out)
    _check_list(d, idx, count, int(S))
    need = lib().lasnet_packed_weights_bytes(LASNET_BF16, int(x.shape[3]), int(M), int(S))
    if need and packed.numel() * packed.element_size() < need:
        raise ValueError("packed buffer too small for this shape")
    if b1.numel() != M or b2.numel() != M or b3.numel() != x.shape[3]:
        raise ValueError("biases: b1 [M], b2 [M], b3 [C]")
    st = lib().lasnet_sparse_bottleneck_packed(ctypes.byref(d), _ptr(idx), _ptr(count), int(S), int(M),
                                               _ptr(packed), _ptr(_f32(b1, "b1")), _ptr(_f32(b2, "b2")),
                                               _ptr(_f32(b3, "b3")), ctypes.byref(o), int(flags),
                                               _stream(stream))
    _check(st, "lasnet_sparse_bottleneck_packed")
    return out


def lasnet_microbench_mfma(iters: int, sink: torch.Tensor, stream=None) -> float:
    """Launches the register-only bf16 MFMA loop; returns the FLOPs of the launch."""
    f = lib().lasnet_microbench_mfma(int(iters), _ptr(sink), _stream(stream))
    if f <= 0:
        raise LasnetError(LASNET_EHIP, "lasnet_microbench_mfma")
    return float(f)


def lasnet_microbench_weight_stream(buf: torch.Tensor, passes: int, sink: torch.Tensor, stream=None) -> float:
    """Every CU reads `buf` `passes` times the way the block kernels read their weights; returns the bytes read."""
    f = lib().lasnet_microbench_weight_stream(_ptr(buf), buf.numel() * buf.element_size(), int(passes), _ptr(sink),
                                              _stream(stream))
    if f <= 0:
        raise LasnetError(LASNET_EHIP, "lasnet_microbench_weight_stream")
    return float(f)


def lasnet_microbench_copy(src: torch.Tensor, dst: torch.Tensor, stream=None) -> int:
    """dst = src with the library's copy kernel; returns the bytes copied."""
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise ValueError("src and dst must have the same size")
    _check(lib().lasnet_microbench_copy(_ptr(src), _ptr(dst), nbytes, _stream(stream)), "lasnet_microbench_copy")
    return nbytes


# ---- rows and experts ----
# Rows are tensors of two dimensions whose rows are dense (their distance is free), or dense tensors of more, whose last dimension
# is a row's: a feature map [N,H,W,C] is N*H*W rows.  8-bit rows are torch.float8_e4m3fn, their scales torch.float8_e8m0fnu (or uint8: the same
# bytes).  A call without an output makes it, as memory of its stream (`stream`, or the current one).

_ROW_DTYPES = {torch.float32: LASNET_F32, torch.bfloat16: LASNET_BF16, torch.float8_e4m3fn: LASNET_E4M3}
_SCALE_DTYPES = (torch.float8_e8m0fnu, torch.uint8)


def _rows(t: Optional[torch.Tensor], name: str) -> Optional[lasnet_rows]:
    if t is None:
        return None
    dt = _ROW_DTYPES.get(t.dtype)
    if dt is None:
        raise ValueError("%s: rows are float32, bfloat16 or float8_e4m3fn" % name)
    if not t.is_cuda:
        raise ValueError("%s: rows live in device memory" % name)
    shape = t.shape
    if len(shape) < 2 or shape[-1] == 0:
        raise ValueError("%s: rows are a tensor [..., cols] of at least two dimensions" % name)
    cols = shape[-1]
    n = t.numel() // cols
    if n <= 1 or t.is_contiguous():
        if n == 1 and cols > 1 and t.stride(-1) != 1:
            raise ValueError("%s: the elements of a row must be contiguous" % name)
        stride = cols
    else:
        if len(shape) != 2 or (cols > 1 and t.stride(1) != 1) or t.stride(0) < cols:
            raise ValueError("%s: rows are dense, and apart from each other, in two dimensions; tensors of more are contiguous" % name)
        stride = t.stride(0)
    return lasnet_rows(t.data_ptr() or None, n, stride, cols, dt)


def _ref(d: Optional[lasnet_rows]):
    return None if d is None else ctypes.byref(d)


def _dense(t: Optional[torch.Tensor], name: str, numel: int, *dtypes) -> Optional[int]:
    """Address of a dense tensor of one of these types and this many elements (None: None)."""
    if t is None:
        return None
    if t.dtype not in dtypes or t.numel() != numel or not t.is_contiguous() or not t.is_cuda:
        raise ValueError("%s must be a contiguous device tensor of %d elements of %s" % (name, numel, " or ".join(str(d) for d in dtypes)))
    return t.data_ptr()


def _workspace(t: Optional[torch.Tensor], need: int, device, stream):
    """(address, bytes, tensor to keep until the call is enqueued)."""
    if t is None and need:
        t = _empty(need, torch.uint8, device, stream)
    elif t is not None and (not t.is_cuda or t.device != device or not t.is_contiguous()):
        raise ValueError("workspace must be a contiguous device tensor, where the rows are")
    return (None, 0, None) if t is None else (t.data_ptr(), t.numel() * t.element_size(), t)


def lasnet_norm_rows(x: torch.Tensor, weight: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                     sum_out: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None,
                     out_dtype: Optional[torch.dtype] = None, stream=None):
    """(out, scale, sum_out): out = s / rms(s) * weight with s = x + residual.  out_dtype (where out is not given): x's, or
    torch.float8_e4m3fn; scale: of 8-bit rows, else None.  sum_out = s, made where there is a residual.  rstd [rows] float32: written where given."""
    if (stream is None and out is not None and out_dtype is None and (sum_out is not None or residual is None)
            and (scale is not None or out.dtype != torch.float8_e4m3fn)):
        L = lib()
        st = _marshal.norm_rows(L.at_norm_rows, x, weight, eps, residual, out, scale, sum_out, rstd)
        if st is not None:
            _check(st, "lasnet_norm_rows")
            return out, scale, sum_out
    d = _rows(x, "x")
    if out is None:
        out = _output(x.shape, out_dtype or x.dtype, x.device, stream)
    elif out_dtype is not None and out.dtype != out_dtype:
        raise ValueError("out has another type than out_dtype")
    if scale is None and out.dtype == torch.float8_e4m3fn:
        scale = _output(d.rows, torch.float8_e8m0fnu, x.device, stream)
    if sum_out is None and residual is not None:
        sum_out = _output(x.shape, x.dtype, x.device, stream)
    r, s, o = _rows(residual, "residual"), _rows(sum_out, "sum_out"), _rows(out, "out")
    st = lib().lasnet_norm_rows(ctypes.byref(d), _ref(r), _dense(weight, "weight", d.cols, torch.float32), eps, _ref(s), ctypes.byref(o),
                                _dense(scale, "scale", d.rows, *_SCALE_DTYPES), _dense(rstd, "rstd", d.rows, torch.float32), _stream(stream))
    _check(st, "lasnet_norm_rows")
    return out, scale, sum_out


def lasnet_norm_rows_backward(dy: torch.Tensor, s: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor,
                              dsum: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                              dweight: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """(dx, dweight) from the gradient dy of lasnet_norm_rows' out and dsum of its sum; s, rstd: as the forward call wrote them."""
    if stream is None and dx is not None and dweight is not None:
        L = lib()
        cols = s.shape[-1] if s.dim() else 0
        need = L.lasnet_norm_rows_backward_workspace_bytes(s.numel() // cols, cols) if cols and workspace is None else 0
        st = _marshal.norm_rows_backward(L.at_norm_rows_backward, dy, s, weight, rstd, dsum, dx, dweight, _workspace(workspace, need, s.device, None)[2])
        if st is not None:
            _check(st, "lasnet_norm_rows_backward")
            return dx, dweight
    y, d, g = _rows(dy, "dy"), _rows(s, "s"), _rows(dsum, "dsum")
    if dx is None:
        dx = _output(s.shape, s.dtype, s.device, stream)
    if dweight is None:
        dweight = _output(d.cols, torch.float32, s.device, stream)
    o, L = _rows(dx, "dx"), lib()
    at, size, keep = _workspace(workspace, L.lasnet_norm_rows_backward_workspace_bytes(d.rows, d.cols), s.device, stream)
    st = L.lasnet_norm_rows_backward(ctypes.byref(y), ctypes.byref(d), _dense(weight, "weight", d.cols, torch.float32),
                                     _dense(rstd, "rstd", d.rows, torch.float32), _ref(g), ctypes.byref(o),
                                     _dense(dweight, "dweight", d.cols, torch.float32), at, size, _stream(stream))
    _check(st, "lasnet_norm_rows_backward")
    return dx, dweight


def lasnet_route(experts: torch.Tensor, E: int, offsets: Optional[torch.Tensor] = None, order: Optional[torch.Tensor] = None,
                 position: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """(offsets [E+1], order [tokens*k], position [tokens,k]), int32, of experts int32 [tokens,k] (outside [0,E): not sent)."""
    if stream is None and offsets is not None and order is not None and position is not None:
        L = lib()
        need = L.lasnet_route_workspace_bytes(experts.shape[0], experts.shape[1], E) if workspace is None and experts.dim() == 2 else 0
        st = _marshal.route(L.at_route, experts, E, offsets, order, position, _workspace(workspace, need, experts.device, None)[2])
        if st is not None:
            _check(st, "lasnet_route")
            return offsets, order, position
    if experts.dim() != 2 or experts.dtype != torch.int32 or not experts.is_cuda or not experts.is_contiguous():
        raise ValueError("experts must be a contiguous int32 device tensor [tokens, k]")
    tokens, k = experts.shape
    if offsets is None:
        offsets = _output(E + 1, torch.int32, experts.device, stream)
    if order is None:
        order = _output(tokens * k, torch.int32, experts.device, stream)
    if position is None:
        position = _output((tokens, k), torch.int32, experts.device, stream)
    L = lib()
    at, size, keep = _workspace(workspace, L.lasnet_route_workspace_bytes(tokens, k, E), experts.device, stream)
    st = L.lasnet_route(_ptr(experts), tokens, k, E, _dense(offsets, "offsets", E + 1, torch.int32), _dense(order, "order", tokens * k, torch.int32),
                        _dense(position, "position", tokens * k, torch.int32), at, size, _stream(stream))
    _check(st, "lasnet_route")
    return offsets, order, position


def _slots(position: torch.Tensor):
    if position.dim() != 2 or position.dtype != torch.int32 or not position.is_cuda or not position.is_contiguous():
        raise ValueError("position must be a contiguous int32 device tensor [tokens, k]")
    return position.shape


def _offsets(offsets: torch.Tensor) -> int:
    if offsets.dim() != 1 or offsets.numel() < 2 or offsets.dtype != torch.int32 or not offsets.is_cuda or not offsets.is_contiguous():
        raise ValueError("offsets must be a contiguous int32 device tensor [E + 1]")
    return offsets.numel() - 1


def lasnet_dispatch_rows(x: torch.Tensor, position: torch.Tensor, offsets: torch.Tensor, scale: Optional[torch.Tensor] = None,
                         out: Optional[torch.Tensor] = None, out_scale: Optional[torch.Tensor] = None, stream=None):
    """(out [tokens*k, cols], out_scale): out[position[t, j]] = x[t], zeros where no expert has a row; the scales of 8-bit rows go along."""
    if stream is None and out is not None and (out_scale is not None or scale is None):
        L = lib()
        st = _marshal.dispatch_rows(L.at_dispatch_rows, x, position, offsets, scale, out, out_scale)
        if st is not None:
            _check(st, "lasnet_dispatch_rows")
            return out, out_scale
    tokens, k = _slots(position)
    E, d = _offsets(offsets), _rows(x, "x")
    if d.rows != tokens:
        raise ValueError("x and position must have as many tokens")
    if out is None:
        out = _output((tokens * k, d.cols), x.dtype, x.device, stream)
    if out_scale is None and scale is not None:
        out_scale = _output(tokens * k, scale.dtype, x.device, stream)
    o = _rows(out, "out")
    st = lib().lasnet_dispatch_rows(ctypes.byref(d), _dense(scale, "scale", tokens, *_SCALE_DTYPES), _ptr(position), _ptr(offsets), k, E,
                                    ctypes.byref(o), _dense(out_scale, "out_scale", tokens * k, *_SCALE_DTYPES), _stream(stream))
    _check(st, "lasnet_dispatch_rows")
    return out, out_scale


def lasnet_combine_rows(y: torch.Tensor, position: torch.Tensor, weights: Optional[torch.Tensor] = None,
                        base: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[t] = base[t] + sum_j weights[t, j] * y[position[t, j]] over the slots that were sent."""
    if stream is None and out is not None:
        L = lib()
        st = _marshal.combine_rows(L.at_combine_rows, y, position, weights, base, out)
        if st is not None:
            _check(st, "lasnet_combine_rows")
            return out
    tokens, k = _slots(position)
    d, b = _rows(y, "y"), _rows(base, "base")
    if out is None:
        out = _output((tokens, d.cols) if base is None else base.shape, y.dtype, y.device, stream)
    o = _rows(out, "out")
    if o.rows != tokens:
        raise ValueError("out and position must have as many tokens")
    st = lib().lasnet_combine_rows(ctypes.byref(d), _dense(weights, "weights", tokens * k, torch.float32), _ptr(position), k, _ref(b),
                                   ctypes.byref(o), _stream(stream))
    _check(st, "lasnet_combine_rows")
    return out


def lasnet_combine_rows_backward(dout: torch.Tensor, y: torch.Tensor, position: torch.Tensor, offsets: torch.Tensor,
                                 weights: Optional[torch.Tensor] = None, dy: Optional[torch.Tensor] = None,
                                 dweights: Optional[torch.Tensor] = None, stream=None):
    """(dy, dweights [tokens, k]) of lasnet_combine_rows; that of base is dout."""
    if stream is None and dy is not None and dweights is not None:
        L = lib()
        st = _marshal.combine_rows_backward(L.at_combine_rows_backward, dout, y, position, offsets, weights, dy, dweights)
        if st is not None:
            _check(st, "lasnet_combine_rows_backward")
            return dy, dweights
    tokens, k = _slots(position)
    E, d, v = _offsets(offsets), _rows(dout, "dout"), _rows(y, "y")
    if d.rows != tokens:
        raise ValueError("dout and position must have as many tokens")
    if dy is None:
        dy = _output(y.shape, y.dtype, y.device, stream)
    if dweights is None:
        dweights = _output((tokens, k), torch.float32, y.device, stream)
    o = _rows(dy, "dy")
    st = lib().lasnet_combine_rows_backward(ctypes.byref(d), ctypes.byref(v), _dense(weights, "weights", tokens * k, torch.float32), _ptr(position),
                                            _ptr(offsets), k, E, ctypes.byref(o), _dense(dweights, "dweights", tokens * k, torch.float32),
                                            _stream(stream))
    _check(st, "lasnet_combine_rows_backward")
    return dy, dweights


def _matrices(W: torch.Tensor, E: int, n: int, k: int, *dtypes) -> Optional[int]:
    if tuple(W.shape) != (E, n, k):
        raise ValueError("the experts' matrices are [%d, %d, %d], not %s" % (E, n, k, tuple(W.shape)))
    return _dense(W, "the experts' matrices", E * n * k, *dtypes)


def lasnet_expert_product(x: torch.Tensor, offsets: torch.Tensor, W: torch.Tensor, scale: Optional[torch.Tensor] = None,
                          wscale: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, flags: int = 0, stream=None) -> torch.Tensor:
    """out[p] = W[e] x[p] for the rows p of each expert e (W [E, n, cols]); bfloat16, or e4m3 with scale [rows], wscale [E, n]."""
    if stream is None and out is not None:
        L = lib()
        st = _marshal.expert_product(L.at_expert_product, x, offsets, W, scale, wscale, out, flags)
        if st is not None:
            _check(st, "lasnet_expert_product")
            return out
    E, d = _offsets(offsets), _rows(x, "x")
    if W.dim() != 3:
        raise ValueError("the experts' matrices are [E, n, cols]")
    n = W.shape[1]
    if out is None:
        out = _output((d.rows, n), torch.bfloat16, x.device, stream)
    o = _rows(out, "out")
    if o.cols != n:
        raise ValueError("out must have %d columns" % n)
    st = lib().lasnet_expert_product(ctypes.byref(d), _dense(scale, "scale", d.rows, *_SCALE_DTYPES), _ptr(offsets), E,
                                     _matrices(W, E, n, d.cols, x.dtype), _dense(wscale, "wscale", E * n, torch.float32), ctypes.byref(o),
                                     flags, _stream(stream))
    _check(st, "lasnet_expert_product")
    return out


def lasnet_expert_product_dx(dy: torch.Tensor, offsets: torch.Tensor, W: torch.Tensor, dx: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dx[p] = W[e]^T dy[p]."""
    if stream is None and dx is not None:
        L = lib()
        st = _marshal.expert_product_dx(L.at_expert_product_dx, dy, offsets, W, dx)
        if st is not None:
            _check(st, "lasnet_expert_product_dx")
            return dx
    E, d = _offsets(offsets), _rows(dy, "dy")
    if W.dim() != 3:
        raise ValueError("the experts' matrices are [E, n, cols]")
    if dx is None:
        dx = _output((d.rows, W.shape[2]), dy.dtype, dy.device, stream)
    o = _rows(dx, "dx")
    st = lib().lasnet_expert_product_dx(ctypes.byref(d), _ptr(offsets), E, _matrices(W, E, d.cols, o.cols, dy.dtype), ctypes.byref(o), _stream(stream))
    _check(st, "lasnet_expert_product_dx")
    return dx


def lasnet_expert_product_dw(dy: torch.Tensor, x: torch.Tensor, offsets: torch.Tensor, dW: Optional[torch.Tensor] = None,
                             dtype: Optional[torch.dtype] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dW[e] = sum over the rows p of expert e of dy[p] x[p]^T; dW [E, n, cols] in bfloat16 (or dtype: float32).  workspace (uint8; made where not given): of
    lasnet_expert_product_dw_workspace_bytes() bytes."""
    L = lib()
    if stream is None and dW is not None and dtype is None:
        rows = x.numel() // max(x.shape[-1], 1) if x.dim() else 0
        need = L.lasnet_expert_product_dw_workspace_bytes(rows, *dW.shape) if workspace is None and rows >= 4096 and dW.dim() == 3 else 0
        st = _marshal.expert_product_dw(L.at_expert_product_dw_ex, dy, x, offsets, dW, _workspace(workspace, need, x.device, None)[2])
        if st is not None:
            _check(st, "lasnet_expert_product_dw_ex")
            return dW
    E, d, v = _offsets(offsets), _rows(dy, "dy"), _rows(x, "x")
    if dW is None:
        dW = _output((E, d.cols, v.cols), dtype or x.dtype, x.device, stream)
    elif dtype is not None and dW.dtype != dtype:
        raise ValueError("dW has another type than dtype")
    at, size, keep = _workspace(workspace, L.lasnet_expert_product_dw_workspace_bytes(v.rows, E, d.cols, v.cols), x.device, stream)
    st = L.lasnet_expert_product_dw_ex(ctypes.byref(d), ctypes.byref(v), _ptr(offsets), E,
                                       _matrices(dW, E, d.cols, v.cols, torch.bfloat16, torch.float32), _ROW_DTYPES[dW.dtype], at, size, _stream(stream))
    _check(st, "lasnet_expert_product_dw_ex")
    return dW


# ---- the router, and products in 8 bits with scales for blocks of 128 ----

def lasnet_choose_experts(logits: torch.Tensor, k: int, mask: Optional[torch.Tensor] = None, experts: Optional[torch.Tensor] = None,
                          weights: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, flags: int = 0, stream=None):
    """(experts int32 [tokens, k], weights [tokens, k], lse [tokens]): each token's k largest of logits [tokens, E], their softmax (LASNET_WEIGHTS_OF_ALL: among all), and
    the logarithm of the sum of exponentials.  mask (uint8 or bool [tokens]): 0, the token takes no part (experts -1)."""
    if stream is None and experts is not None and weights is not None and lse is not None:
        L = lib()
        st = _marshal.choose_experts(L.at_choose_experts, logits, mask, k, experts, weights, lse, flags)
        if st is not None:
            _check(st, "lasnet_choose_experts")
            return experts, weights, lse
    d = _rows(logits, "logits")
    if k > 0:
        if experts is None:
            experts = _output((d.rows, k), torch.int32, logits.device, stream)
        if weights is None:
            weights = _output((d.rows, k), torch.float32, logits.device, stream)
    if lse is None:
        lse = _output(d.rows, torch.float32, logits.device, stream)
    st = lib().lasnet_choose_experts(ctypes.byref(d), _dense(mask, "mask", d.rows, torch.uint8, torch.bool), k, _dense(experts, "experts", d.rows * k, torch.int32),
                                     _dense(weights, "weights", d.rows * k, torch.float32), _dense(lse, "lse", d.rows, torch.float32), flags, _stream(stream))
    _check(st, "lasnet_choose_experts")
    return experts, weights, lse


def _chosen(experts: torch.Tensor) -> int:
    if experts.dim() != 2 or experts.dtype != torch.int32 or not experts.is_cuda or not experts.is_contiguous():
        raise ValueError("experts must be a contiguous int32 device tensor [tokens, k]")
    return experts.shape[1]


def lasnet_balance(logits: torch.Tensor, lse: torch.Tensor, experts: torch.Tensor, counts: Optional[torch.Tensor] = None, share: Optional[torch.Tensor] = None,
                   loss: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """(counts int32 [E + 1], share [E], loss [2]): rows of each expert (and, last, the tokens that took part), mean probabilities, the balance loss and the mean of lse^2.
    experts: as lasnet_route gets them (-1: a slot that was dropped)."""
    L = lib()
    if stream is None and counts is not None and share is not None and loss is not None:
        E = logits.shape[-1] if logits.dim() >= 2 else 0
        need = L.lasnet_balance_workspace_bytes(logits.numel() // E, E) if E and workspace is None else 0
        st = _marshal.balance(L.at_balance, logits, lse, experts, counts, share, loss, _workspace(workspace, need, logits.device, None)[2])
        if st is not None:
            _check(st, "lasnet_balance")
            return counts, share, loss
    d, k = _rows(logits, "logits"), _chosen(experts)
    if counts is None:
        counts = _output(d.cols + 1, torch.int32, logits.device, stream)
    if share is None:
        share = _output(d.cols, torch.float32, logits.device, stream)
    if loss is None:
        loss = _output(2, torch.float32, logits.device, stream)
    at, size, keep = _workspace(workspace, L.lasnet_balance_workspace_bytes(d.rows, d.cols), logits.device, stream)
    st = L.lasnet_balance(ctypes.byref(d), _dense(lse, "lse", d.rows, torch.float32), _dense(experts, "experts", d.rows * k, torch.int32), k,
                          _dense(counts, "counts", d.cols + 1, torch.int32), _dense(share, "share", d.cols, torch.float32),
                          _dense(loss, "loss", 2, torch.float32), at, size, _stream(stream))
    _check(st, "lasnet_balance")
    return counts, share, loss


def lasnet_choose_experts_backward(logits: torch.Tensor, lse: torch.Tensor, experts: torch.Tensor, weights: torch.Tensor, dweights: Optional[torch.Tensor] = None,
                                   counts: Optional[torch.Tensor] = None, dloss: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None,
                                   flags: int = 0, stream=None) -> torch.Tensor:
    """dlogits (as logits) from the gradient dweights of the weights and dloss [2] of lasnet_balance's loss (with its counts).  experts, weights: as chosen, slots that were dropped
    afterwards included (their dweights are 0)."""
    if stream is None and dlogits is not None:
        L = lib()
        st = _marshal.choose_experts_backward(L.at_choose_experts_backward, logits, lse, experts, weights, dweights, counts, dloss, dlogits, flags)
        if st is not None:
            _check(st, "lasnet_choose_experts_backward")
            return dlogits
    d, k = _rows(logits, "logits"), _chosen(experts)
    if dlogits is None:
        dlogits = _output(logits.shape, logits.dtype, logits.device, stream)
    o = _rows(dlogits, "dlogits")
    st = lib().lasnet_choose_experts_backward(ctypes.byref(d), _dense(lse, "lse", d.rows, torch.float32), _dense(experts, "experts", d.rows * k, torch.int32),
                                              _dense(weights, "weights", d.rows * k, torch.float32), k, _dense(dweights, "dweights", d.rows * k, torch.float32),
                                              _dense(counts, "counts", d.cols + 1, torch.int32), _dense(dloss, "dloss", 2, torch.float32), ctypes.byref(o),
                                              flags, _stream(stream))
    _check(st, "lasnet_choose_experts_backward")
    return dlogits


def _blocks(n: int) -> int:
    return (n + 127) // 128


def lasnet_quantize_rows(x: torch.Tensor, position: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                         scale: Optional[torch.Tensor] = None, stream=None):
    """(out e4m3, scale [rows, ceil(cols / 128)]): x in 8 bits with a scale for each 128 columns; with position and offsets laid out by expert, as lasnet_dispatch_rows does."""
    if stream is None and out is not None and scale is not None:
        L = lib()
        st = _marshal.quantize_rows(L.at_quantize_rows, x, position, offsets, out, scale)
        if st is not None:
            _check(st, "lasnet_quantize_rows")
            return out, scale
    d = _rows(x, "x")
    if (position is None) != (offsets is None):
        raise ValueError("position and offsets come together")
    if position is None:
        k, E, rows = 1, 1, d.rows
    else:
        tokens, k = _slots(position)
        E, rows = _offsets(offsets), tokens * k
        if d.rows != tokens:
            raise ValueError("x and position must have as many tokens")
    if out is None:
        out = _output(x.shape if position is None else (rows, d.cols), torch.float8_e4m3fn, x.device, stream)
    if scale is None:
        scale = _output((rows, _blocks(d.cols)), torch.float8_e8m0fnu, x.device, stream)
    o = _rows(out, "out")
    st = lib().lasnet_quantize_rows(ctypes.byref(d), _ptr(position), _ptr(offsets), k, E, ctypes.byref(o),
                                    _dense(scale, "scale", rows * _blocks(d.cols), *_SCALE_DTYPES), _stream(stream))
    _check(st, "lasnet_quantize_rows")
    return out, scale


def lasnet_quantize_matrices(W: torch.Tensor, transposed: bool = False, out: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                             out_t: Optional[torch.Tensor] = None, scale_t: Optional[torch.Tensor] = None, stream=None):
    """(out e4m3 [E, n, k], scale [E, ceil(n / 128), ceil(k / 128)], out_t [E, k, n], scale_t): the experts' matrices in 8 bits with a scale for each block of 128 x 128.
    transposed: makes the last two, too (else None, where they are not given)."""
    if stream is None and out is not None and scale is not None and (not transposed or (out_t is not None and scale_t is not None)):
        L = lib()
        st = _marshal.quantize_matrices(L.at_quantize_matrices, W, out, scale, out_t, scale_t)
        if st is not None:
            _check(st, "lasnet_quantize_matrices")
            return out, scale, out_t, scale_t
    if W.dim() != 3 or W.dtype not in _DTYPES:
        raise ValueError("the experts' matrices are float32 or bfloat16 [E, n, k]")
    E, n, k = W.shape
    if (out_t is None) != (scale_t is None):
        raise ValueError("out_t and scale_t come together")
    if out is None:
        out = _output((E, n, k), torch.float8_e4m3fn, W.device, stream)
    if scale is None:
        scale = _output((E, _blocks(n), _blocks(k)), torch.float8_e8m0fnu, W.device, stream)
    if out_t is None and transposed:
        out_t = _output((E, k, n), torch.float8_e4m3fn, W.device, stream)
        scale_t = _output((E, _blocks(k), _blocks(n)), torch.float8_e8m0fnu, W.device, stream)
    cells = E * _blocks(n) * _blocks(k)
    st = lib().lasnet_quantize_matrices(_matrices(W, E, n, k, W.dtype), _DTYPES[W.dtype], E, n, k, _matrices(out, E, n, k, torch.float8_e4m3fn),
                                        _dense(scale, "scale", cells, *_SCALE_DTYPES), None if out_t is None else _matrices(out_t, E, k, n, torch.float8_e4m3fn),
                                        _dense(scale_t, "scale_t", cells, *_SCALE_DTYPES), _stream(stream))
    _check(st, "lasnet_quantize_matrices")
    return out, scale, out_t, scale_t


def lasnet_block_product(x: torch.Tensor, scale: torch.Tensor, offsets: torch.Tensor, W: torch.Tensor, wscale: torch.Tensor,
                         out: Optional[torch.Tensor] = None, flags: int = 0, stream=None) -> torch.Tensor:
    """out[p] = W[e] x[p] for the rows p of each expert e: e4m3 rows with scale [rows, ceil(cols / 128)] and matrices [E, n, cols] with wscale
    [E, ceil(n / 128), ceil(cols / 128)] (e8m0 as lasnet_quantize_matrices writes them, or float32); out bfloat16."""
    if stream is None and out is not None:
        L = lib()
        st = _marshal.block_product(L.at_block_product, x, scale, offsets, W, wscale, out, flags)
        if st is not None:
            _check(st, "lasnet_block_product")
            return out
    E, d = _offsets(offsets), _rows(x, "x")
    if W.dim() != 3:
        raise ValueError("the experts' matrices are [E, n, cols]")
    n = W.shape[1]
    if out is None:
        out = _output((d.rows, n), torch.bfloat16, x.device, stream)
    o = _rows(out, "out")
    if o.cols != n:
        raise ValueError("out must have %d columns" % n)
    st = lib().lasnet_block_product(ctypes.byref(d), _dense(scale, "scale", d.rows * _blocks(d.cols), *_SCALE_DTYPES), _ptr(offsets), E,
                                    _matrices(W, E, n, d.cols, x.dtype), _dense(wscale, "wscale", E * _blocks(n) * _blocks(d.cols), torch.float32, *_SCALE_DTYPES),
                                    LASNET_F32 if wscale.dtype == torch.float32 else LASNET_E8M0, ctypes.byref(o), flags, _stream(stream))
    _check(st, "lasnet_block_product")
    return out

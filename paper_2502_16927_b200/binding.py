"""ctypes binding of libbigmac's C ABI (include/bigmac.h): same names, argument marshalling only.

Every step of the layer runs inside the library's CUDA kernels; torch is used here for device
memory and streams.  There is no fallback: if the shared library is missing or a call fails, an
exception is raised.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
import struct
from typing import Dict, NamedTuple, Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libbigmac.so")

BIGMAC_OK = 0
BIGMAC_F32, BIGMAC_BF16 = 0, 1
BIGMAC_FLAG_SIMT_GEMM = 1


class bigmac_config_t(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("d", "r", "h", "E", "k", "max_tokens", "dtype", "act")] + [("flags", C.c_uint32)] +
                [("capacity_factor", C.c_double), ("aux_loss_coef", C.c_double)])


class bigmac_weights_t(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w_gate", "b_gate", "w_down", "w1", "w2", "w_up", "b1", "b2")]


class bigmac_grads_t(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("dw_gate", "db_gate", "dw_down", "dw1", "dw2", "dw_up", "db1", "db2")]


_ROUTING_FIELDS = ("topk_idx", "topk_w", "counts", "offsets", "row_of_slot", "slot_of_row", "counts_chosen", "aux_loss")


class bigmac_routing_t(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _ROUTING_FIELDS]


class bigmac_debug_gemm_t(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("A", "B", "C", "Z")] + [(n, C.c_int64) for n in ("lda", "ldb", "ldc")] +
                [(n, C.c_int32) for n in ("M", "N", "K", "a_kmajor", "b_kmajor", "out_f32", "accumulate", "epilogue",
                                          "act", "group", "num_experts")] +
                [(n, C.c_int64) for n in ("b_stride", "c_stride")] +
                [(n, C.c_void_p) for n in ("tile_expert", "n_tiles", "poffsets")])


BIGMAC_PROFILE_SLOTS = 32


class bigmac_profile_t(C.Structure):
    _fields_ = [("launches", C.c_uint64), ("dropped", C.c_uint32), ("n_slots", C.c_int32),
                ("ms", C.c_float * BIGMAC_PROFILE_SLOTS), ("calls", C.c_uint32 * BIGMAC_PROFILE_SLOTS)]


BIGMAC_EP_MAX_RANKS = 8


class bigmac_ep_t(C.Structure):
    _fields_ = [("rank", C.c_int32), ("size", C.c_int32), ("counts_all", C.c_void_p)] + \
               [(n, C.c_void_p * BIGMAC_EP_MAX_RANKS) for n in ("xg", "u", "du", "dxg")]




class bigmac_mx4_t(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p)] + [(n, C.c_int32) for n in ("rows", "K", "E")] + [("offsets", C.c_void_p)]


_lib: Optional[C.CDLL] = None


def lib() -> C.CDLL:
    """Load libbigmac.so (built in-tree by paper_2502_16927_b200/build.py); raises if it is absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2502_16927_b200.build` first")
        L = C.CDLL(LIB_PATH)
        vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        L.bigmac_layer_create.argtypes = [C.POINTER(bigmac_config_t), C.POINTER(vp)]
        L.bigmac_layer_destroy.argtypes = [vp]
        L.bigmac_workspace_bytes.argtypes = [vp, i32, C.c_int, C.POINTER(sz), C.POINTER(sz)]
        L.bigmac_route.argtypes = [vp, vp, i32, C.POINTER(bigmac_weights_t), C.POINTER(bigmac_routing_t), vp, sz, vp]
        L.bigmac_forward.argtypes = [vp, vp, i32, C.POINTER(bigmac_weights_t), vp, C.POINTER(bigmac_routing_t), vp,
                                     vp, sz, vp]
        L.bigmac_backward.argtypes = [vp, vp, vp, i32, C.POINTER(bigmac_weights_t), vp, vp, C.POINTER(bigmac_grads_t),
                                      C.c_int, vp, sz, vp]
        L.bigmac_device_status.argtypes = [vp, vp]
        L.bigmac_status_string.argtypes = [C.c_int]
        L.bigmac_status_string.restype = C.c_char_p
        L.bigmac_exchange_rows.argtypes = [vp, vp, i32, i32, vp, vp, sz, vp, C.c_int, vp]
        L.bigmac_debug_gemm.argtypes = [vp, C.POINTER(bigmac_debug_gemm_t), C.c_int, vp]
        L.bigmac_debug_expire_wait.argtypes = [vp, vp]
        L.bigmac_debug_expire_wait.restype = C.c_int
        L.bigmac_debug_decode_launches.argtypes = [vp, C.c_uint32, vp]
        L.bigmac_debug_decode_launches.restype = C.c_int
        L.bigmac_debug_set.argtypes = [C.c_char_p, C.c_int]
        L.bigmac_debug_set.restype = C.c_int
        L.bigmac_route_static.argtypes = [vp, vp, i32, C.POINTER(bigmac_weights_t), C.POINTER(bigmac_routing_t), vp]
        L.bigmac_route_static.restype = C.c_int
        L.bigmac_profile_enable.argtypes = [vp, C.c_int]
        L.bigmac_profile_read.argtypes = [vp, vp, C.POINTER(bigmac_profile_t)]
        L.bigmac_profile_slot_name.argtypes = [C.c_int]
        L.bigmac_profile_slot_name.restype = C.c_char_p
        W, R, G, EP = (C.POINTER(t) for t in (bigmac_weights_t, bigmac_routing_t, bigmac_grads_t, bigmac_ep_t))
        L.bigmac_ep_buffer_bytes.argtypes = [vp, i32, C.POINTER(sz)]
        L.bigmac_ep_workspace_bytes.argtypes = [vp, i32, i32, C.POINTER(sz), C.POINTER(sz)]
        L.bigmac_ep_route.argtypes = [vp, vp, i32, W, EP, R, vp, vp, sz, vp]
        L.bigmac_ep_dispatch.argtypes = [vp, i32, EP, vp, vp]
        L.bigmac_ep_experts.argtypes = [vp, W, EP, vp, vp]
        L.bigmac_ep_combine.argtypes = [vp, i32, W, EP, vp, vp, vp]
        L.bigmac_ep_backward_combine.argtypes = [vp, vp, i32, W, EP, G, C.c_int, vp, vp, sz, vp]
        L.bigmac_ep_backward_experts.argtypes = [vp, W, EP, G, C.c_int, vp, vp, sz, vp]
        L.bigmac_ep_backward_dispatch.argtypes = [vp, vp, i32, W, EP, vp, G, C.c_int, vp, vp, sz, vp]
        Q, i64 = C.POINTER(bigmac_mx4_t), C.c_int64
        L.bigmac_operator_status.argtypes = [vp]
        L.bigmac_mx4_bytes.argtypes = [i32, i32, i32, C.c_int, C.POINTER(sz), C.POINTER(sz)]
        L.bigmac_mx4_quantize.argtypes = [vp, i32, i32, i64, vp, i32, Q, vp]
        L.bigmac_mx4_dequantize.argtypes = [Q, vp, i32, i64, vp]
        L.bigmac_mx4_matmul.argtypes = [Q, Q, i32, i32, vp, i64, vp]
        L.bigmac_mx4_matmul_mx4.argtypes = [Q, Q, i32, Q, vp]
        L.bigmac_mx4_matmul_mx4.restype = C.c_int
        L.bigmac_mx4_workspace_bytes.argtypes = [vp, i32, C.POINTER(sz)]
        L.bigmac_mx4_workspace_bytes.restype = C.c_int
        L.bigmac_forward_mx4.argtypes = [vp, vp, i32, C.POINTER(bigmac_weights_t), Q, Q, vp, C.POINTER(bigmac_routing_t), vp, sz, vp]
        L.bigmac_forward_mx4.restype = C.c_int
        L.bigmac_residual_norm_forward.argtypes = [vp, i32, vp]
        L.bigmac_residual_norm_scratch_bytes.argtypes = [vp, i32, C.POINTER(sz)]
        L.bigmac_residual_norm_backward.argtypes = [vp, i32, C.c_int, vp, sz, vp]
        for name in ("bigmac_residual_norm_forward", "bigmac_residual_norm_scratch_bytes", "bigmac_residual_norm_backward",
                     "bigmac_operator_status", "bigmac_mx4_bytes", "bigmac_mx4_quantize", "bigmac_mx4_dequantize", "bigmac_mx4_matmul"):
            getattr(L, name).restype = C.c_int
        for name in ("bigmac_ep_buffer_bytes", "bigmac_ep_workspace_bytes", "bigmac_ep_route", "bigmac_ep_dispatch",
                     "bigmac_ep_experts", "bigmac_ep_combine", "bigmac_ep_backward_combine", "bigmac_ep_backward_experts",
                     "bigmac_ep_backward_dispatch"):
            getattr(L, name).restype = C.c_int
        for name in ("bigmac_profile_enable", "bigmac_profile_read", "bigmac_layer_create", "bigmac_layer_destroy", "bigmac_workspace_bytes", "bigmac_route",
                     "bigmac_forward", "bigmac_backward", "bigmac_device_status", "bigmac_exchange_rows",
                     "bigmac_debug_gemm"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


class BigmacError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib().bigmac_status_string(status).decode()} ({status})")


def _check(status: int, where: str) -> None:
    if status != BIGMAC_OK:
        raise BigmacError(status, where)


# The marshalling sits in front of every launch, and for one decoded token it took longer than the kernel (14 us of Python
# around 5 us in the library): addresses are passed as plain integers, and the stream handle comes from the accessor that
# builds no Stream object (0.1 us against 3.3).

def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "tensors passed to libbigmac must be contiguous CUDA tensors"
    return t.data_ptr()


_raw_stream, _current_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream() -> int:
    if _raw_stream is None or _current_device is None:      # a torch that has the two accessors under other names
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_current_device())


# ---- the C ABI, name for name -------------------------------------------------------------------------

def bigmac_layer_create(d, r, h, E, k, max_tokens, dtype, act, flags=0, capacity_factor=0.0, aux_loss_coef=0.0) -> C.c_void_p:
    cfg = bigmac_config_t(d, r, h, E, k, max_tokens, dtype, act, flags, capacity_factor, aux_loss_coef)
    handle = C.c_void_p()
    _check(lib().bigmac_layer_create(C.byref(cfg), C.byref(handle)), "bigmac_layer_create")
    return handle


def bigmac_layer_destroy(handle) -> None:
    _check(lib().bigmac_layer_destroy(handle), "bigmac_layer_destroy")


def bigmac_workspace_bytes(handle, T: int, training: bool):
    s, v = C.c_size_t(), C.c_size_t()
    _check(lib().bigmac_workspace_bytes(handle, T, int(training), C.byref(s), C.byref(v)), "bigmac_workspace_bytes")
    return s.value, v.value


def _weights(W: Dict[str, torch.Tensor]) -> bigmac_weights_t:
    # w_down / w_up are absent for the projection-free layer (BIGMAC_FLAG_CDAC)
    get = W.get
    return bigmac_weights_t(_ptr(get("w_gate")), _ptr(get("b_gate")), _ptr(get("w_down")), _ptr(get("w1")),
                            _ptr(get("w2")), _ptr(get("w_up")), _ptr(get("b1")), _ptr(get("b2")))


def _grads(G: Dict[str, torch.Tensor]) -> bigmac_grads_t:
    return bigmac_grads_t(*[_ptr(G.get(n)) for n in ("dw_gate", "db_gate", "dw_down", "dw1", "dw2", "dw_up", "db1", "db2")])


def _routing(R: Optional[Dict[str, torch.Tensor]]):
    if R is None:
        return None
    return C.byref(bigmac_routing_t(*[_ptr(R.get(n)) for n in _ROUTING_FIELDS]))


def bigmac_route(handle, x, T, W, routing, scratch) -> None:
    _check(lib().bigmac_route(handle, _ptr(x), T, C.byref(_weights(W)), _routing(routing), _ptr(scratch),
                              scratch.numel() * scratch.element_size(), _stream()), "bigmac_route")


def bigmac_route_static(handle, x, T, W, routing) -> None:
    """bigmac_route without a scratch buffer: intermediates live in the library's fixed device array
    (BIGMAC_STATIC_SCRATCH_BYTES).  For callers that cannot allocate device memory; raises BigmacError with
    status -7 if (T, E, k) does not fit.  Calls must not overlap on the GPU (they share the array)."""
    _check(lib().bigmac_route_static(handle, _ptr(x), T, C.byref(_weights(W)), _routing(routing), _stream()),
           "bigmac_route_static")


def bigmac_forward(handle, x, T, W, y, routing, saved, scratch) -> None:
    _check(lib().bigmac_forward(handle, _ptr(x), T, C.byref(_weights(W)), _ptr(y), _routing(routing), _ptr(saved),
                                _ptr(scratch), scratch.numel() * scratch.element_size(), _stream()), "bigmac_forward")


def bigmac_backward(handle, x, dy, T, W, saved, dx, G, accumulate, scratch) -> None:
    _check(lib().bigmac_backward(handle, _ptr(x), _ptr(dy), T, C.byref(_weights(W)), _ptr(saved), _ptr(dx),
                                 C.byref(_grads(G)), int(accumulate), _ptr(scratch),
                                 scratch.numel() * scratch.element_size(), _stream()), "bigmac_backward")


def bigmac_device_status(handle) -> int:
    return lib().bigmac_device_status(handle, _stream())


def bigmac_exchange_rows(handle, saved, T, width, src, grouped, dst, which) -> None:
    _check(lib().bigmac_exchange_rows(handle, _ptr(saved), T, width, _ptr(src), _ptr(grouped),
                                      grouped.numel() * grouped.element_size(), _ptr(dst), which, _stream()),
           "bigmac_exchange_rows")


def bigmac_profile_enable(handle, on: bool) -> None:
    _check(lib().bigmac_profile_enable(handle, int(on)), "bigmac_profile_enable")


def bigmac_profile_read(handle) -> Dict[str, object]:
    """Synchronises the current stream; returns {"launches", "dropped", "stages": {name: (ms, calls)}}."""
    prof = bigmac_profile_t()
    _check(lib().bigmac_profile_read(handle, _stream(), C.byref(prof)), "bigmac_profile_read")
    stages = {lib().bigmac_profile_slot_name(i).decode(): (float(prof.ms[i]), int(prof.calls[i]))
              for i in range(prof.n_slots) if prof.calls[i]}
    return {"launches": int(prof.launches), "dropped": int(prof.dropped), "stages": stages}


def bigmac_debug_gemm(handle, q: bigmac_debug_gemm_t, use_tensor_cores) -> None:
    """use_tensor_cores: False/0 plain FMA, True/1 tensor cores, 2 one-CTA kernel, 3/4/5 CTA-pair kernel with 4/2/1 working
    epilogue warps per lane quadrant."""
    _check(lib().bigmac_debug_gemm(handle, C.byref(q), int(use_tensor_cores), _stream()), "bigmac_debug_gemm")


def bigmac_debug_set(name: str, value: int = 0) -> None:
    """Process-wide measurement / debugging switch ("overlap", "tc_pair", "groupk", "ffn", "fused_mlp", "epi_parts",
    "staged_stores", "fuse_dispatch", "mx4_tile", "tc_mask"; "defaults" restores all).  The defaults are the product."""
    _check(lib().bigmac_debug_set(name.encode(), int(value)), "bigmac_debug_set")


def bigmac_debug_expire_wait(handle) -> None:
    """Launch the one-thread kernel whose bounded wait runs out (failure path of the device-side waits)."""
    _check(lib().bigmac_debug_expire_wait(handle, _stream()), "bigmac_debug_expire_wait")


def bigmac_debug_decode_launches(handle, launches: int) -> None:
    """Set the launch count of the small-batch kernel's memory (the tags of its hand-over words go on from there)."""
    _check(lib().bigmac_debug_decode_launches(handle, launches, _stream()), "bigmac_debug_decode_launches")


# ---- expert parallelism: the phase calls, name for name ----------------------------------------------------

def bigmac_ep_buffer_bytes(handle, size: int) -> int:
    n = C.c_size_t()
    _check(lib().bigmac_ep_buffer_bytes(handle, size, C.byref(n)), "bigmac_ep_buffer_bytes")
    return n.value


def bigmac_ep_workspace_bytes(handle, T: int, size: int):
    s, v = C.c_size_t(), C.c_size_t()
    _check(lib().bigmac_ep_workspace_bytes(handle, T, size, C.byref(s), C.byref(v)), "bigmac_ep_workspace_bytes")
    return s.value, v.value


def make_ep(rank: int, size: int, counts_all: torch.Tensor, ptrs: Dict[str, list]) -> bigmac_ep_t:
    """ptrs[name][q]: device address (int) of rank q's exchange buffer `name` as this rank addresses it."""
    ep = bigmac_ep_t()
    ep.rank, ep.size, ep.counts_all = rank, size, counts_all.data_ptr()
    for name in ("xg", "u", "du", "dxg"):
        arr = getattr(ep, name)
        for q in range(size):
            arr[q] = ptrs[name][q]
    return ep


def _nbytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def bigmac_ep_route(handle, x, T, W, ep, routing, saved, scratch) -> None:
    _check(lib().bigmac_ep_route(handle, _ptr(x), T, C.byref(_weights(W)), C.byref(ep), _routing(routing), _ptr(saved),
                                 _ptr(scratch), _nbytes(scratch), _stream()), "bigmac_ep_route")


def bigmac_ep_dispatch(handle, T, ep, saved) -> None:
    _check(lib().bigmac_ep_dispatch(handle, T, C.byref(ep), _ptr(saved), _stream()), "bigmac_ep_dispatch")


def bigmac_ep_experts(handle, W, ep, saved) -> None:
    _check(lib().bigmac_ep_experts(handle, C.byref(_weights(W)), C.byref(ep), _ptr(saved), _stream()), "bigmac_ep_experts")


def bigmac_ep_combine(handle, T, W, ep, y, saved) -> None:
    _check(lib().bigmac_ep_combine(handle, T, C.byref(_weights(W)), C.byref(ep), _ptr(y), _ptr(saved), _stream()),
           "bigmac_ep_combine")


def bigmac_ep_backward_combine(handle, dy, T, W, ep, G, accumulate, saved, scratch) -> None:
    _check(lib().bigmac_ep_backward_combine(handle, _ptr(dy), T, C.byref(_weights(W)), C.byref(ep), C.byref(_grads(G)),
                                            int(accumulate), _ptr(saved), _ptr(scratch), _nbytes(scratch), _stream()),
           "bigmac_ep_backward_combine")


def bigmac_ep_backward_experts(handle, W, ep, G, accumulate, saved, scratch) -> None:
    _check(lib().bigmac_ep_backward_experts(handle, C.byref(_weights(W)), C.byref(ep), C.byref(_grads(G)), int(accumulate),
                                            _ptr(saved), _ptr(scratch), _nbytes(scratch), _stream()),
           "bigmac_ep_backward_experts")


def bigmac_ep_backward_dispatch(handle, x, T, W, ep, dx, G, accumulate, saved, scratch) -> None:
    _check(lib().bigmac_ep_backward_dispatch(handle, _ptr(x), T, C.byref(_weights(W)), C.byref(ep), _ptr(dx),
                                             C.byref(_grads(G)), int(accumulate), _ptr(saved), _ptr(scratch),
                                             _nbytes(scratch), _stream()), "bigmac_ep_backward_dispatch")


# ---- operators around the layer ----------------------------------------------------------------------------

def operator_status() -> int:
    """Synchronises the current stream; 0, or the error that a kernel of the calls below recorded since the last look."""
    return lib().bigmac_operator_status(_stream())


_DTYPES = {torch.float32: BIGMAC_F32, torch.bfloat16: BIGMAC_BF16}


def _dtype(t: torch.dtype) -> int:
    try:
        return _DTYPES[t]
    except KeyError:
        raise ValueError(f"{t}: float32 and bfloat16 are supported") from None


def _here() -> int:
    """The current device: the kernels run on it, whatever device a tensor is on."""
    return _current_device() if _current_device is not None else torch.cuda.current_device()


@functools.lru_cache(maxsize=None)
def _device(index: int) -> torch.device:
    return torch.device("cuda", index)


_MOST_ROWS = 0x7fffffff                                 # int32_t of the C calls


def _dense(t: torch.Tensor, name: str, here: int) -> int:
    if t.get_device() != here or here < 0 or not t.is_contiguous():
        raise ValueError(f"{name}: a dense tensor on the current device, cuda:{here}, is needed")
    return t.data_ptr()


def _matrix(t: torch.Tensor, shape, name: str, here: int):
    """(address, row stride) of a matrix with dense rows; shape is t.shape."""
    if t.get_device() == here and len(shape) == 2 and shape[0] <= _MOST_ROWS:
        if t.is_contiguous():
            return t.data_ptr(), shape[1]
        rows, columns = shape
        ld, step = t.stride()
        if (step == 1 or columns == 1) and (ld >= columns or rows == 1):
            return t.data_ptr(), max(ld, columns)
    raise ValueError(f"{name}: a matrix with dense rows (2^31 - 1 at most) that do not overlap, on the current device, cuda:{here}, is needed")


def _new(rows: int, columns: int, dtype, device) -> torch.Tensor:
    return torch.empty_strided((rows, columns), (columns, 1), dtype=dtype, device=device)       # half the time of torch.empty


def _vector(t: Optional[torch.Tensor], name: str, n: int, here: int) -> int:
    if t is None:
        return 0
    if t.dtype is not torch.float32 or t.dim() != 1 or t.shape[0] != n:
        raise ValueError(f"{name}: an fp32 vector of {n} is needed")
    return _dense(t, name, here)


BIGMAC_NORM_NONE, BIGMAC_NORM_RMS, BIGMAC_NORM_LAYER = 0, 1, 2
BIGMAC_GATE_NONE, BIGMAC_GATE_TOKEN, BIGMAC_GATE_CHANNEL, BIGMAC_GATE_FULL = 0, 1, 2, 3


class Norm(NamedTuple):
    """A norm of the joint (bigmac_norm_t) with its fp32 parameters [d]; None: ones, zeros."""
    kind: int
    weight: Optional[torch.Tensor] = None
    bias: Optional[torch.Tensor] = None
    eps: float = 1e-6


_NO_NORM = Norm(BIGMAC_NORM_NONE)
# bigmac_residual_norm_t, packed at once: a ctypes structure of as many members takes longer to fill than a token's kernel runs
_RESIDUAL_NORM = struct.Struct("@5i3f4P" + 5 * "Pq" + "P" + 5 * "Pq" + "4P")
_NOTHING = (0, 0)
_NO_BACKWARD = 14 * (0,)


def _rows_like(t: Optional[torch.Tensor], name: str, shape, dtype, here: int):
    """(address, row stride) of a matrix of this shape and type, (0, 0) where there is none."""
    if t is None:
        return _NOTHING
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name}: {tuple(shape)} of {dtype} is needed, not {tuple(t.shape)} of {t.dtype}")
    return _matrix(t, shape, name, here)


def _gate_kind(gate, T: int, gate_kind) -> int:
    """The gate's kind by its shape; a vector as long as both T and d is one factor a token unless gate_kind says otherwise."""
    if gate.dim() == 2:
        kind = BIGMAC_GATE_FULL
    elif gate_kind == BIGMAC_GATE_TOKEN or gate_kind == BIGMAC_GATE_CHANNEL:
        return gate_kind
    else:
        kind = BIGMAC_GATE_TOKEN if gate.shape[0] == T else BIGMAC_GATE_CHANNEL
    if gate_kind is not None and kind != gate_kind:
        raise ValueError(f"gate_kind {gate_kind}: a gate of shape {tuple(gate.shape)}")
    return kind


def _joint(x, shape, dtype, y, gate, gate_kind, post, pre, residual_scale, here):
    """The members of bigmac_residual_norm_t that forward and backward share, up to `gate`."""
    at, ld = _matrix(x, shape, "x", here)
    T, d = shape
    kind, g = BIGMAC_GATE_NONE, _NOTHING
    if gate is not None:
        kind = _gate_kind(gate, T, gate_kind)
        g = _rows_like(gate, "gate", shape, dtype, here) if kind == BIGMAC_GATE_FULL else (_vector(gate, "gate", T if kind == BIGMAC_GATE_TOKEN else d, here), 0)
    post_kind, w_post, b_post, post_eps = _NO_NORM if post is None else post
    pre_kind, w_pre, b_pre, pre_eps = _NO_NORM if pre is None else pre
    return (d, _dtype(dtype), post_kind, pre_kind, kind, post_eps, pre_eps, residual_scale, _vector(w_post, "post.weight", d, here),
            _vector(b_post, "post.bias", d, here), _vector(w_pre, "pre.weight", d, here), _vector(b_pre, "pre.bias", d, here), at, ld,
            *_rows_like(y, "y", shape, dtype, here), *g)


def residual_norm_forward(x: torch.Tensor, y: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None, post: Optional[Norm] = None,
                          pre: Optional[Norm] = None, residual_scale: float = 1.0, training: bool = False, gate_kind: Optional[int] = None,
                          r: Optional[torch.Tensor] = None, n: Optional[torch.Tensor] = None, want_r: bool = True):
    """r = residual_scale x + gate N_post(y) and n = N_pre(r) (bigmac_residual_norm_forward): (r, n, stats), n None without `pre`, stats (for
    the backward) None unless `training`.  gate: [T] or [d] fp32, or [T, d].  r and n may be given, in place too (r is x, n is y); r is
    neither written nor returned without want_r."""
    here, shape, dtype = _here(), x.shape, x.dtype
    members = _joint(x, shape, dtype, y, gate, gate_kind, post, pre, residual_scale, here)
    T, d = shape
    if r is None and want_r:
        r = torch.empty_like(x)
        r_at, r_ld = r.data_ptr(), d
    else:
        r_at, r_ld = _rows_like(r, "r", shape, dtype, here)
    if n is None and members[3] != BIGMAC_NORM_NONE:
        n = torch.empty_like(x)
        n_at, n_ld = n.data_ptr(), d
    else:
        n_at, n_ld = _rows_like(n, "n", shape, dtype, here)
    stats = _new(T, 4, torch.float32, x.device) if training else None
    q = _RESIDUAL_NORM.pack(*members, r_at, r_ld, n_at, n_ld, 0 if stats is None else stats.data_ptr(), *_NO_BACKWARD)
    _check(lib().bigmac_residual_norm_forward(q, T, _stream()), "bigmac_residual_norm_forward")
    return r, n, stats


_residual_norm_scratch = {}                             # bytes by (device, T, d): a function of the sizes and the card


def residual_norm_backward(x, y, gate, post, pre, dr, dn, stats, G: Optional[Dict[str, torch.Tensor]] = None, residual_scale: float = 1.0,
                           accumulate: bool = False, gate_kind: Optional[int] = None):
    """Gradients of sum(r dr) + sum(n dn) (bigmac_residual_norm_backward): (dx, dy, dgate), None for what was not in the call.  G holds
    fp32 buffers for the gradients of the parameters, any of dw_post, db_post, dw_pre, db_pre and, for a gate [d], dgate (returned,
    too); with `accumulate` they are added to.  dr or dn may be None."""
    here, shape, dtype = _here(), x.shape, x.dtype
    members = _joint(x, shape, dtype, y, gate, gate_kind, post, pre, residual_scale, here)
    T, d = shape
    kind = members[4]
    dx = torch.empty_like(x)
    dy_at, dy_ld, dy = 0, 0, None
    if y is not None:
        dy = torch.empty_like(x)
        dy_at, dy_ld = dy.data_ptr(), d
    grads = [0, 0, 0, 0]
    if G:
        get = G.get
        grads = [_vector(get("dw_post"), "dw_post", d, here), _vector(get("db_post"), "db_post", d, here),
                 _vector(get("dw_pre"), "dw_pre", d, here), _vector(get("db_pre"), "db_pre", d, here)]
    dgate, dg_at, dg_ld = None, 0, 0
    if kind == BIGMAC_GATE_CHANNEL:
        dgate = G.get("dgate") if G else None
        dg_at = _vector(dgate, "dgate", d, here)
    elif kind != BIGMAC_GATE_NONE:
        dgate = torch.empty_like(gate)
        dg_at, dg_ld = dgate.data_ptr(), d
    if stats is None or stats.dtype is not torch.float32 or stats.shape != (T, 4):
        raise ValueError("stats: those of a training forward of the same rows")
    q = _RESIDUAL_NORM.pack(*members, 0, 0, 0, 0, _dense(stats, "stats", here), *_rows_like(dr, "dr", shape, dtype, here),
                            *_rows_like(dn, "dn", shape, dtype, here), dx.data_ptr(), d, dy_at, dy_ld, dg_at, dg_ld, *grads)
    scratch, at, need = None, None, 0
    if any(grads) or (kind == BIGMAC_GATE_CHANNEL and dg_at):
        need = _residual_norm_scratch.get((here, T, d))
        if need is None:
            size = C.c_size_t()
            _check(lib().bigmac_residual_norm_scratch_bytes(q, T, C.byref(size)), "bigmac_residual_norm_scratch_bytes")
            if len(_residual_norm_scratch) >= 4096:
                _residual_norm_scratch.clear()
            need = _residual_norm_scratch[here, T, d] = size.value
        if need:
            scratch = torch.empty_strided((need,), (1,), dtype=torch.uint8, device=x.device)
            at = scratch.data_ptr()
    _check(lib().bigmac_residual_norm_backward(q, T, accumulate, at, need, _stream()), "bigmac_residual_norm_backward")
    return dx, dy, dgate


class Mx4:
    """A matrix in microscaled 4-bit floating point (bigmac_mx4_t): codes [rows, K / 2] and scales [row tiles, K tiles, 512] of one
    matrix, both with a leading E for the stacked weights of E experts; with `offsets` (int32 [E + 1]) the segments of a routing's
    experts, `rows` rows in the caller's order."""
    __slots__ = ("_codes", "_scales", "_room", "offsets", "rows", "_c", "_device")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, offsets: Optional[torch.Tensor] = None, rows: Optional[int] = None):
        shape = codes.shape
        stored, half, E = shape[-2] if len(shape) > 1 else 0, shape[-1], shape[0] if len(shape) == 3 else 0
        tiles = (-(-stored // 128), -(-half // 64), 512)
        if (codes.dtype is not torch.uint8 or scales.dtype is not torch.uint8 or not 1 < len(shape) < 4 or
                scales.shape != (tiles if len(shape) == 2 else (E, *tiles))):
            raise ValueError(f"Mx4: codes [rows, K / 2] and scales [row tiles, K tiles, 512] of torch.uint8, or both with a leading E; not "
                             f"{tuple(shape)} and {tuple(scales.shape)}")
        device, table = codes.get_device(), None
        if offsets is None:
            rows = stored
        else:
            if E or rows is None:
                raise ValueError("a grouped Mx4 has codes of two dimensions and rows")
            E, table = _offsets(offsets, device), offsets.data_ptr()
            if stored < _mx4_stored(rows, E):
                raise ValueError(f"Mx4: {rows} rows of {E} experts need {_mx4_stored(rows, E)} rows of codes")
        if not 0 <= rows <= _MOST_ROWS:
            raise ValueError(f"Mx4: {rows} rows")
        self._codes, self._scales, self._room, self.offsets, self.rows, self._device = codes, scales, None, offsets, rows, device
        self._c = bigmac_mx4_t(_dense(codes, "codes", device), _dense(scales, "scales", device), rows, 2 * half, E, table)

    @classmethod
    def _empty(cls, stored: int, rows: int, K: int, offsets, E: int, table, device, here: int) -> "Mx4":
        """Room for a result: one allocation, codes and scales as tensors only when they are asked for."""
        q = cls.__new__(cls)
        code_bytes = stored * (K // 2)
        q._room = torch.empty_strided((code_bytes + -(-stored // 128) * -(-K // 128) * 512,), (1,), dtype=torch.uint8, device=device)
        at = q._room.data_ptr()
        q._codes = q._scales = None
        q.offsets, q.rows, q._device = offsets, rows, here
        q._c = bigmac_mx4_t(at, at + code_bytes, rows, K, E, table)
        return q

    def _views(self):
        half = self._c.K // 2
        stored = _mx4_stored(self.rows, self._c.E) if self.offsets is not None else self.rows
        self._codes = self._room[:stored * half].view(stored, half)
        self._scales = self._room[stored * half:].view(-(-stored // 128), -(-half // 64), 512)

    @property
    def codes(self) -> torch.Tensor:
        if self._codes is None:
            self._views()
        return self._codes

    @property
    def scales(self) -> torch.Tensor:
        if self._scales is None:
            self._views()
        return self._scales


def _mx4(q: Mx4, here: int) -> bigmac_mx4_t:
    if q._device != here:
        raise ValueError(f"Mx4 on cuda:{q._device}, the current device is cuda:{here}")
    return q._c


def _mx4_stored(rows: int, E: int) -> int:
    """Rows that a grouped matrix has room for: each expert's segment begins at a multiple of 128."""
    return (rows + min(rows, E) * 127) // 128 * 128


def _offsets(t: torch.Tensor, here: int) -> int:
    """The number of experts of a table of segments."""
    if t.dtype is not torch.int32 or t.dim() != 1 or t.shape[0] < 2:
        raise ValueError("offsets: an int32 vector [E + 1] is needed")
    _dense(t, "offsets", here)
    return t.shape[0] - 1


def mx4_quantize(x: torch.Tensor, offsets: Optional[torch.Tensor] = None, slot_of_row: Optional[torch.Tensor] = None, k: int = 1) -> Mx4:
    """Rows of x to 4 bits (bigmac_mx4_quantize).  With `offsets` (int32 [E + 1], of a routing) grouped by expert; with `slot_of_row`
    row i is x[slot_of_row[i] // k]: the dispatch."""
    here, shape = _here(), x.shape
    ptr, ld = _matrix(x, shape, "x", here)
    x_rows, K = shape
    rows, slots, E, table = x_rows, None, 0, None
    if K == 0 or K % 32:
        raise ValueError(f"K = {K}: blocks of 32 columns")
    if slot_of_row is not None:
        if slot_of_row.dtype is not torch.int32 or slot_of_row.dim() != 1 or slot_of_row.shape[0] > _MOST_ROWS:
            raise ValueError("slot_of_row: an int32 vector is needed")
        slots, rows = _dense(slot_of_row, "slot_of_row", here), slot_of_row.shape[0]
    stored = rows
    if offsets is not None:
        E, table = _offsets(offsets, here), offsets.data_ptr()
        stored = _mx4_stored(rows, E)
    q = Mx4._empty(stored, rows, K, offsets, E, table, x.device, here)
    _check(lib().bigmac_mx4_quantize(ptr, _dtype(x.dtype), x_rows, ld, slots, k, C.byref(q._c), _stream()), "bigmac_mx4_quantize")
    return q


def _output(out, rows: int, columns: int, dtype, here: int):
    """The result's matrix: (tensor, address, row stride, bigmac_dtype_t)."""
    if out is None:
        out = _new(rows, columns, dtype, _device(here))
        return out, out.data_ptr(), columns, _dtype(dtype)
    if out.shape != (rows, columns):
        raise ValueError(f"out has shape {tuple(out.shape)}, not {(rows, columns)}")
    return (out, *_matrix(out, out.shape, "out", here), _dtype(out.dtype))


def mx4_dequantize(q: Mx4, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The numbers a matrix stands for, in the caller's order of rows.  Of a grouped one, rows in no segment keep what `out` holds."""
    here = _here()
    c = _mx4(q, here)
    out, ptr, ld, kind = _output(out, c.rows, c.K, dtype, here)
    _check(lib().bigmac_mx4_dequantize(C.byref(c), ptr, kind, ld, _stream()), "bigmac_mx4_dequantize")
    return out


def mx4_matmul(a: Mx4, w: Mx4, act: int = 3, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """act(a w^T) (bigmac_mx4_matmul; act a bigmac_act_t, 3 the identity).  For a grouped `a`, `w` holds the matrices of its experts."""
    here = _here()
    ca, cw = _mx4(a, here), _mx4(w, here)
    out, ptr, ld, kind = _output(out, ca.rows, cw.rows, dtype, here)
    _check(lib().bigmac_mx4_matmul(C.byref(ca), C.byref(cw), act, kind, ptr, ld, _stream()), "bigmac_mx4_matmul")
    return out


def mx4_matmul_mx4(a: Mx4, w: Mx4, act: int = 3) -> Mx4:
    """act(a w^T) in 4 bits (bigmac_mx4_matmul_mx4), with a's rows: the input of a next product."""
    here = _here()
    ca, cw = _mx4(a, here), _mx4(w, here)
    if cw.rows == 0 or cw.rows % 32:
        raise ValueError(f"{cw.rows} columns: blocks of 32")
    stored = ca.rows if a.offsets is None else _mx4_stored(ca.rows, ca.E)
    out = Mx4._empty(stored, ca.rows, cw.rows, a.offsets, ca.E, ca.offsets, _device(here), here)
    _check(lib().bigmac_mx4_matmul_mx4(C.byref(ca), C.byref(cw), act, C.byref(out._c), _stream()), "bigmac_mx4_matmul_mx4")
    return out


def mx4_quantize_weights(w: torch.Tensor) -> Mx4:
    """The stacked weights [E, N, K] of E experts, laid out once."""
    if w.dim() != 3:
        raise ValueError("w: [E, N, K]")
    parts = [mx4_quantize(one) for one in w]
    return Mx4(torch.stack([q.codes for q in parts]), torch.stack([q.scales for q in parts]))


def bigmac_mx4_workspace_bytes(handle, T: int) -> int:
    n = C.c_size_t()
    _check(lib().bigmac_mx4_workspace_bytes(handle, T, C.byref(n)), "bigmac_mx4_workspace_bytes")
    return n.value


def bigmac_forward_mx4(handle, x, T, W, w1: Mx4, w2: Mx4, y, routing, scratch) -> None:
    here = _here()
    _check(lib().bigmac_forward_mx4(handle, _ptr(x), T, C.byref(_weights(W)), C.byref(_mx4(w1, here)), C.byref(_mx4(w2, here)), _ptr(y), _routing(routing),
                                    _ptr(scratch), scratch.numel() * scratch.element_size(), _stream()), "bigmac_forward_mx4")


# ---- a small convenience wrapper: owns the handle and the workspaces ------------------------------------

class Layer:
    """One BigMac layer handle plus torch-allocated workspaces.  Marshalling only."""

    def __init__(self, d, r, h, E, k, max_tokens, dtype, act, flags=0, device="cuda", capacity_factor=0.0, aux_loss_coef=0.0):
        self.cfg = dict(d=d, r=r, h=h, E=E, k=k, max_tokens=max_tokens, dtype=dtype, act=act, flags=flags,
                        capacity_factor=capacity_factor, aux_loss_coef=aux_loss_coef)
        self.device = torch.device(device)
        with torch.cuda.device(self.device):
            self.handle = bigmac_layer_create(d, r, h, E, k, max_tokens, dtype, act, flags, capacity_factor, aux_loss_coef)
        self.tdtype = torch.bfloat16 if dtype == BIGMAC_BF16 else torch.float32
        self._scratch = None
        self._saved = None
        self._need = {}
        self._T = None
        self._steps = 0                                 # training forwards so far

    def close(self):
        if self.handle is not None:
            bigmac_layer_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _workspaces(self, T, training):
        need = self._need.get((T, training))
        if need is None:                                # a function of the handle's configuration, T and the direction
            if len(self._need) >= 4096:
                self._need.clear()
            need = self._need[(T, training)] = bigmac_workspace_bytes(self.handle, T, training)
        s, v = need
        if self._scratch is None or self._scratch.numel() < s:
            self._scratch = torch.empty(max(s, 256), dtype=torch.uint8, device=self.device)
        if training and (self._saved is None or self._saved.numel() < v):
            self._saved = torch.empty(max(v, 256), dtype=torch.uint8, device=self.device)

    def empty_routing(self, T):
        # Two allocations and splits instead of eight allocations (13 us), every table on a 16-byte boundary.  The tables of the slots
        # are apart from those of the experts: a program that keeps the loss or the loads of a step keeps a few KB with it.
        E, n = self.cfg["E"], T * self.cfg["k"]
        nn, ee = n + -n % 4, E + -E % 4
        empty = functools.partial(torch.empty, dtype=torch.int32, device=self.device)
        idx, w, row, slot = empty(4 * nn).split_with_sizes([nn, nn, nn, nn])
        counts, chosen, aux, _, offsets = empty(3 * ee + 5).split_with_sizes([ee, ee, 1, 3, ee + 1])
        if nn != n:
            idx, w, row, slot = idx[:n], w[:n], row[:n], slot[:n]
        if ee != E:
            counts, chosen, offsets = counts[:E], chosen[:E], offsets[:E + 1]
        return {"topk_idx": idx, "topk_w": w.view(torch.float32), "counts": counts, "offsets": offsets, "row_of_slot": row,
                "slot_of_row": slot, "counts_chosen": chosen, "aux_loss": aux.view(torch.float32)}

    def route(self, x, W):
        T = x.shape[0]
        self._workspaces(T, False)
        R = self.empty_routing(T)
        bigmac_route(self.handle, x, T, W, R, self._scratch)
        return R

    def _check_tokens(self, t, name):
        """The kernels take a handle's width and type for granted: anything else would be read, or written, past its end."""
        if t.dim() != 2 or t.shape[1] != self.cfg["d"] or t.dtype is not self.tdtype:
            raise ValueError(f"{name}: [T, {self.cfg['d']}] of {self.tdtype} is needed, not {tuple(t.shape)} of {t.dtype}")

    def _forward_mx4(self, x, W, y, want_routing):
        """The inference forward with experts in 4 bits."""
        self._check_tokens(x, "x")
        if y is not None:
            self._check_tokens(y, "y")
            if y.shape != x.shape:
                raise ValueError(f"y has shape {tuple(y.shape)}, not {tuple(x.shape)}")
        T = x.shape[0]
        need = self._need.get((T, "mx4"))
        if need is None:
            if len(self._need) >= 4096:
                self._need.clear()
            need = self._need[T, "mx4"] = bigmac_mx4_workspace_bytes(self.handle, T)
        if self._scratch is None or self._scratch.numel() < need:
            self._scratch = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        if y is None:
            y = torch.empty_like(x)
        R = self.empty_routing(T) if want_routing else None
        shared = {name: t for name, t in W.items() if name not in ("w1", "w2")}
        bigmac_forward_mx4(self.handle, x, T, shared, W["w1"], W["w2"], y, R, self._scratch)
        self._T = None
        return (y, R) if want_routing else y

    def forward(self, x, W, y=None, training=False, want_routing=False):
        """W: the weights by name; w1 and w2 as `Mx4` (mx4_quantize_weights) run the experts in 4 bits (inference only)."""
        if isinstance(W.get("w1"), Mx4) or isinstance(W.get("w2"), Mx4):
            if training or not (isinstance(W["w1"], Mx4) and isinstance(W["w2"], Mx4)):
                raise ValueError("experts in 4 bits: both w1 and w2, inference only")
            return self._forward_mx4(x, W, y, want_routing)
        T = x.shape[0]
        self._workspaces(T, training)
        if y is None:
            y = torch.empty_like(x)
        R = self.empty_routing(T) if want_routing else None
        bigmac_forward(self.handle, x, T, W, y, R, self._saved if training else None, self._scratch)
        self._T = T if training else None
        self._steps += training
        return (y, R) if want_routing else y

    def backward(self, x, dy, W, G, dx=None, accumulate=False):
        T = x.shape[0]
        if self._T != T:
            raise RuntimeError("backward needs a training forward of the same batch first")
        if dx is None:
            dx = torch.empty_like(x)
        bigmac_backward(self.handle, x, dy, T, W, self._saved, dx, G, accumulate, self._scratch)
        return dx

    def status(self) -> int:
        return bigmac_device_status(self.handle)


class Block:
    """The layer as a residual block: out = residual_scale x + gate N_post(layer(N_pre(x))), forward and backward, with the two joints of
    residual_norm_forward around it.  pre, post: `Norm`s (post may be None); gate: a vector of parameters [d], or None.  A backward follows
    the training forward whose gradients it gives: the layer keeps one step."""

    def __init__(self, layer: Layer, pre: Norm, post: Optional[Norm] = None, gate: Optional[torch.Tensor] = None, residual_scale: float = 1.0):
        if pre is None or pre.kind == BIGMAC_NORM_NONE:
            raise ValueError("pre: a block begins with a norm")
        self.layer, self.pre, self.post, self.gate, self.residual_scale = layer, pre, post, gate, residual_scale
        self._gate_kind = None if gate is None else BIGMAC_GATE_CHANNEL
        self._kept = None

    def forward(self, x, W, training=False, want_routing=False):
        self.layer._check_tokens(x, "x")
        _, n, before = residual_norm_forward(x, pre=self.pre, training=training, want_r=False)
        y = self.layer.forward(n, W, training=training, want_routing=want_routing)
        y, R = y if want_routing else (y, None)
        out, _, after = residual_norm_forward(x, y, self.gate, self.post, residual_scale=self.residual_scale, training=training, gate_kind=self._gate_kind)
        self._kept = (x, n, y, before, after, self.layer._steps) if training else None
        return (out, R) if want_routing else out

    def backward(self, dout, W, G, accumulate=False):
        """dx; G: the layer's gradient buffers and, of the block's own parameters, any of dw_pre, db_pre, dw_post, db_post (fp32 [d]) and
        dgate, each a vector of its own (norms that share a parameter, too)."""
        if self._kept is None:
            raise RuntimeError("backward needs a training forward first")
        x, n, y, before, after, step = self._kept
        if step != self.layer._steps or self.layer._T != x.shape[0]:   # before the first launch: it writes gradients
            raise RuntimeError("the layer keeps one step: another forward of it came between")
        here, vectors = _here(), [(name, G[name]) for name in ("dw_pre", "db_pre", "dw_post", "db_post", "dgate") if G.get(name) is not None]
        # two calls write them: one would overwrite the other's
        if len({_vector(t, name, x.shape[1], here) for name, t in vectors}) < len(vectors):
            raise ValueError("two gradients in one place")
        own = {name: G[name] for name in ("dw_post", "db_post", "dgate") if name in G}
        dx, dy, _ = residual_norm_backward(x, y, self.gate, self.post, None, dout, None, after, own, self.residual_scale, accumulate, self._gate_kind)
        dn = self.layer.backward(n, dy, W, G, accumulate=accumulate)
        # the gradient through the norm joins the residual's
        own = {name: G[name] for name in ("dw_pre", "db_pre") if name in G}
        dx, _, _ = residual_norm_backward(x, None, None, None, self.pre, dx, dn, before, own, accumulate=accumulate)
        return dx

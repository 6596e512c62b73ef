"""Thin ctypes binding of ``libmoemix.so``: same names as the C-ABI in ``include/moemix.h``.

Argument marshalling only.  Tensors are ``torch`` CUDA tensors used as device
memory (``data_ptr()``) and the current torch stream is passed through; every
step of the MoE block runs inside the library's kernels.  There is no fallback:
if the library is not built, :func:`lib` raises.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from pathlib import Path
from typing import List, Optional, Sequence

_LIB_PATH = Path(__file__).resolve().parent / "libmoemix.so"

MOE_OK, MOE_EINVAL, MOE_ESHAPE, MOE_ENOTRESIDENT, MOE_EWORKSPACE, MOE_EHIP = 0, -1, -2, -3, -4, -5
PREC_FP16, PREC_INT4G64, PREC_INT8G64, PREC_FP8B128 = 0, 1, 2, 3
GROUP = 64
FP8_BLOCK = 128
OUT_F32, OUT_F16 = 0, 1
MAX_EXPERTS = 32
MAX_GRADS = 1024
STATUS_BAD_INDEX = 1 << 1
STATUS_NOT_RESIDENT = 1 << 3

EXPORTS = (
    "moe_workspace_bytes", "moe_route", "moe_permute", "moe_expert_ffn_mixed", "moe_layer_forward",
    "moe_chain_forward", "moe_dequant_int4", "moe_quantize_int4", "moe_synth_fill_f16", "moe_read_status",
    "moe_last_error", "moe_version", "moe_trace_kernel", "moe_plan", "moe_swap_slot_bytes", "moe_layer_forward_swap",
    "moe_stream_read", "moe_static_scratch_bytes", "moe_layer_forward_static",
    "moe_dequant_int8", "moe_quantize_int8", "moe_quantize_fp8", "moe_dequant_fp8", "moe_quantize_fp8_rows",
    "moe_transpose_fp8", "moe_matmul_fp8", "moe_matmul_fp8_grouped", "moe_route_logits", "moe_gate_workspace_bytes",
    "moe_balance_loss", "moe_route_backward", "moe_experts_workspace_bytes", "moe_experts_forward", "moe_experts_backward",
    "moe_clip_workspace_bytes", "moe_clip_gradients",
)


class MoeError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"moemix error {code}: {msg}")
        self.code = code


class CMat(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("zero", ctypes.c_void_p)]


class CExpert(ctypes.Structure):
    _fields_ = [("prec", ctypes.c_int32), ("resident", ctypes.c_int32), ("w1", CMat), ("w3", CMat), ("w2", CMat)]


class CLayer(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int32), ("d_ff", ctypes.c_int32), ("n_experts", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("w_gate", ctypes.c_void_p), ("gate_bias", ctypes.c_void_p),
                ("experts", ctypes.POINTER(CExpert))]


class CPlanRequest(ctypes.Structure):
    _fields_ = [("mem_gpu", ctypes.c_uint64), ("size_non_expert", ctypes.c_uint64), ("size_e16", ctypes.c_uint64),
                ("size_e4", ctypes.c_uint64), ("swap_bytes", ctypes.c_uint64), ("seed", ctypes.c_uint64),
                ("num_experts", ctypes.c_int32), ("preference", ctypes.c_int32), ("num_e4", ctypes.c_int32)]


class CPlanResult(ctypes.Structure):
    _fields_ = [("num_e16", ctypes.c_int32), ("num_e4", ctypes.c_int32), ("resident_e16", ctypes.c_int32),
                ("resident_e4", ctypes.c_int32), ("bytes_resident", ctypes.c_uint64)]


class CSwap(ctypes.Structure):
    _fields_ = [("host_experts", ctypes.POINTER(CExpert)), ("swap", ctypes.c_void_p), ("slot_bytes", ctypes.c_size_t),
                ("n_slots", ctypes.c_int32), ("host_idx", ctypes.c_void_p), ("copy_stream", ctypes.c_void_p),
                ("copied_event", ctypes.c_void_p), ("computed_event", ctypes.c_void_p)]


class CExpertGrads(ctypes.Structure):
    _fields_ = [("w1", ctypes.c_void_p), ("w3", ctypes.c_void_p), ("w2", ctypes.c_void_p)]


class CGrad(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_size_t), ("grad_type", ctypes.c_int32),
                ("out_type", ctypes.c_int32)]


PREFER_THROUGHPUT, PREFER_QUALITY = 0, 1

_lib = None


def lib():
    """The loaded HIP library.  Raises if it has not been built: there is no other path."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise RuntimeError(f"{_LIB_PATH} is missing: run __graft_entry__.build() (hipcc, gfx950) first")
        # torch first: its HIP runtime owns the streams and the memory that are passed in, and the library
        # must bind to that same runtime instance rather than load a second one
        import torch  # noqa: F401
        L = ctypes.CDLL(str(_LIB_PATH))
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        LP = ctypes.POINTER(CLayer)
        L.moe_workspace_bytes.argtypes = [LP, i32]
        L.moe_workspace_bytes.restype = sz
        L.moe_route.argtypes = [LP, vp, i32, vp, vp, vp]
        L.moe_permute.argtypes = [LP, vp, i32, vp, vp, vp, vp, sz, vp]
        L.moe_expert_ffn_mixed.argtypes = [LP, i32, vp, i32, vp, vp, sz, vp]
        L.moe_layer_forward.argtypes = [LP, vp, i32, vp, vp, vp, vp, sz, vp]
        L.moe_chain_forward.argtypes = [LP, ctypes.POINTER(vp), i32, ctypes.c_float, vp, i32, vp, vp, sz, vp]
        L.moe_dequant_int4.argtypes = [ctypes.POINTER(CMat), i32, i32, vp, vp]
        L.moe_quantize_int4.argtypes = [vp, i32, i32, vp, vp, vp, vp]
        L.moe_dequant_int8.argtypes = [ctypes.POINTER(CMat), i32, i32, vp, vp]
        L.moe_quantize_int8.argtypes = [vp, i32, i32, vp, vp, vp, vp]
        MP = ctypes.POINTER(CMat)
        L.moe_quantize_fp8.argtypes = [vp, i32, i32, vp, vp, vp]
        L.moe_dequant_fp8.argtypes = [MP, i32, i32, vp, vp]
        L.moe_quantize_fp8_rows.argtypes = [vp, i32, i32, vp, vp, vp]
        L.moe_transpose_fp8.argtypes = [MP, i32, i32, vp, vp, vp]
        L.moe_matmul_fp8.argtypes = [MP, i32, i32, vp, vp, i32, vp, i32, vp]
        L.moe_matmul_fp8_grouped.argtypes = [MP, i32, i32, i32, vp, vp, i32, vp, vp, i32, i32, vp, i32, vp]
        L.moe_route_logits.argtypes = [LP, vp, i32, vp, vp, vp, vp]
        L.moe_gate_workspace_bytes.argtypes = [LP, i32]
        L.moe_gate_workspace_bytes.restype = sz
        L.moe_balance_loss.argtypes = [LP, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.moe_route_backward.argtypes = [LP, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.moe_experts_workspace_bytes.argtypes = [LP, i32]
        L.moe_experts_workspace_bytes.restype = sz
        L.moe_experts_forward.argtypes = [LP, vp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.moe_experts_backward.argtypes = [LP, vp, i32, vp, vp, vp, vp, vp, vp, vp, i32, vp, ctypes.POINTER(CExpertGrads), i32, i32, vp, sz, vp]
        L.moe_clip_workspace_bytes.argtypes = [i32]
        L.moe_clip_workspace_bytes.restype = sz
        L.moe_clip_gradients.argtypes = [ctypes.POINTER(CGrad), i32, ctypes.c_float, ctypes.c_float, vp, vp, sz, vp]
        L.moe_synth_fill_f16.argtypes = [vp, sz, sz, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_float, i32, vp]
        L.moe_read_status.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_int)]
        L.moe_trace_kernel.argtypes = [i32, vp, vp]
        L.moe_plan.argtypes = [ctypes.POINTER(CPlanRequest), ctypes.POINTER(CPlanResult), vp, vp]
        L.moe_swap_slot_bytes.argtypes = [LP]
        L.moe_swap_slot_bytes.restype = sz
        L.moe_layer_forward_swap.argtypes = [LP, ctypes.POINTER(CSwap), vp, i32, vp, vp, vp, vp, sz, vp,
                                             ctypes.POINTER(ctypes.c_int32)]
        L.moe_stream_read.argtypes = [vp, sz, vp, vp]
        L.moe_static_scratch_bytes.argtypes = []
        L.moe_static_scratch_bytes.restype = sz
        L.moe_layer_forward_static.argtypes = [LP, vp, i32, vp, vp, vp, vp]
        L.moe_last_error.restype = ctypes.c_char_p
        L.moe_version.restype = i32
        for name in EXPORTS:
            if name not in ("moe_workspace_bytes", "moe_last_error", "moe_version", "moe_swap_slot_bytes",
                            "moe_static_scratch_bytes", "moe_gate_workspace_bytes", "moe_experts_workspace_bytes",
                            "moe_clip_workspace_bytes"):
                getattr(L, name).restype = i32
        _lib = L
    return _lib


def _check(rc: int) -> None:
    if rc != MOE_OK:
        raise MoeError(rc, lib().moe_last_error().decode())


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream() -> int:
    import torch
    return torch.cuda.current_stream().cuda_stream


# ---------------------------------------------------------------- descriptors

@dataclass
class Mat:
    """One weight matrix in device memory: fp16 ``data`` [out,in], uint8 ``data`` [out,in/2] + fp16 scale/zero, or e4m3 ``data`` [out,in]
    (uint8 or float8_e4m3fn) + fp32 ``scale`` [ceil(out/128),ceil(in/128)]."""
    data: "torch.Tensor"
    scale: Optional["torch.Tensor"] = None
    zero: Optional["torch.Tensor"] = None

    def c(self) -> CMat:
        return CMat(_ptr(self.data), _ptr(self.scale), _ptr(self.zero))

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.data, self.scale, self.zero) if t is not None)


@dataclass
class Expert:
    prec: int
    w1: Optional[Mat]
    w3: Optional[Mat]
    w2: Optional[Mat]
    resident: bool = True

    def c(self) -> CExpert:
        null = CMat(None, None, None)
        return CExpert(self.prec, int(self.resident), self.w1.c() if self.w1 else null,
                       self.w3.c() if self.w3 else null, self.w2.c() if self.w2 else null)

    def nbytes(self) -> int:
        return sum(m.nbytes() for m in (self.w1, self.w3, self.w2) if m is not None)


def _fits_fp8(m: Optional[Mat], what: str, out: int, inn: int) -> None:
    """The kernels read what an e4m3 expert's descriptor and its layer's shape say: codes [out,in], fp32 scales per block of 128 x 128."""
    import torch
    blocks = ((out + FP8_BLOCK - 1) // FP8_BLOCK, (inn + FP8_BLOCK - 1) // FP8_BLOCK)
    for t, part, types, shape in ((m and m.data, "codes", (torch.uint8, torch.float8_e4m3fn), (out, inn)), (m and m.scale, "scales", (torch.float32,), blocks)):
        if t is None:
            raise MoeError(MOE_EINVAL, f"{what}: no {part}")
        if t.dtype not in types or not t.is_contiguous():
            raise MoeError(MOE_EINVAL, f"{part} of {what}: {t.dtype}, strides {t.stride()}: contiguous {types} is needed")
        if tuple(t.shape) != shape:
            raise MoeError(MOE_ESHAPE, f"{part} of {what}: {tuple(t.shape)}, {shape} is needed")


def _fitting_expert(e: Expert, prec: int, i: int, d: int, f: int, on_gpu: bool) -> CExpert:
    """C descriptor of expert ``i``, whose matrices fit its layer if they are e4m3 (a missing expert may have none)."""
    if prec == PREC_FP8B128 and (on_gpu or e.w1 or e.w3 or e.w2):
        for m, name, out, inn in ((e.w1, "w1", f, d), (e.w3, "w3", f, d), (e.w2, "w2", d, f)):
            _fits_fp8(m, f"expert {i}, {name}", out, inn)
        if on_gpu and not all(t.is_cuda for m in (e.w1, e.w3, e.w2) for t in (m.data, m.scale)):
            raise MoeError(MOE_EINVAL, f"expert {i} is resident, and not on a GPU")
    return e.c()


class Layer:
    """Host descriptor of one MoE block; keeps the tensors alive that its device pointers name."""

    def __init__(self, d_model: int, d_ff: int, top_k: int, w_gate, experts: Sequence[Expert], gate_bias=None):
        self.d_model, self.d_ff, self.top_k = d_model, d_ff, top_k
        self.w_gate, self.gate_bias, self.experts = w_gate, gate_bias, list(experts)
        self._arr = (CExpert * len(self.experts))(*[_fitting_expert(e, e.prec, i, d_model, d_ff, e.resident) for i, e in enumerate(self.experts)])
        self.c = CLayer(d_model, d_ff, len(self.experts), top_k, _ptr(w_gate), _ptr(gate_bias), self._arr)

    @property
    def n_experts(self) -> int:
        return len(self.experts)


def workspace_bytes(layer: Layer, n_tokens: int, any_precision: bool = False) -> int:
    """``any_precision``: enough for every table of experts of the layer's shape, not for the one it has alone."""
    c = layer.c
    if any_precision:
        c = CLayer(c.d_model, c.d_ff, c.n_experts, c.top_k, c.w_gate, c.gate_bias, None)
    return int(lib().moe_workspace_bytes(ctypes.byref(c), n_tokens))


def alloc_workspace(layer: Layer, n_tokens: int, any_precision: bool = False):
    import torch
    n = workspace_bytes(layer, n_tokens, any_precision)
    if n == 0:
        raise MoeError(MOE_EINVAL, "moe_workspace_bytes rejected the arguments")
    return torch.empty(n, dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------- entry points (same names as the C-ABI)

def moe_route(layer: Layer, x, topk_idx, topk_gate) -> None:
    _check(lib().moe_route(ctypes.byref(layer.c), _ptr(x), x.shape[0], _ptr(topk_idx), _ptr(topk_gate), _stream()))


def moe_permute(layer: Layer, topk_idx, counts, offsets, perm, ws) -> None:
    _check(lib().moe_permute(ctypes.byref(layer.c), _ptr(topk_idx), topk_idx.shape[0], _ptr(counts), _ptr(offsets),
                             _ptr(perm), _ptr(ws), ws.numel(), _stream()))


def moe_expert_ffn_mixed(layer: Layer, expert: int, x_rows, y, ws) -> None:
    _check(lib().moe_expert_ffn_mixed(ctypes.byref(layer.c), expert, _ptr(x_rows), x_rows.shape[0], _ptr(y), _ptr(ws),
                                      0 if ws is None else ws.numel(), _stream()))


def moe_layer_forward(layer: Layer, x, out, ws, topk_idx_out=None, topk_gate_out=None) -> None:
    _check(lib().moe_layer_forward(ctypes.byref(layer.c), _ptr(x), x.shape[0], _ptr(out), _ptr(topk_idx_out),
                                   _ptr(topk_gate_out), _ptr(ws), 0 if ws is None else ws.numel(), _stream()))


def moe_static_scratch_bytes() -> int:
    return int(lib().moe_static_scratch_bytes())


def moe_layer_forward_static(layer: Layer, x, out, topk_idx_out=None, topk_gate_out=None) -> None:
    _check(lib().moe_layer_forward_static(ctypes.byref(layer.c), _ptr(x), x.shape[0], _ptr(out), _ptr(topk_idx_out),
                                          _ptr(topk_gate_out), _stream()))


class Swap:
    """Swap space and host-side expert copies for moe_layer_forward_swap.  `host_experts[e]` is an Expert whose
    tensors are pinned host tensors (or None for experts that are resident in `layer`)."""

    def __init__(self, layer: Layer, host_experts: Sequence[Optional[Expert]], n_slots: int, n_tokens: int):
        import torch
        self.layer, self.host_experts, self.n_slots = layer, list(host_experts), n_slots
        null = CExpert(PREC_FP16, 0, CMat(None, None, None), CMat(None, None, None), CMat(None, None, None))
        self._arr = (CExpert * layer.n_experts)(*[null if e is None else _fitting_expert(e, layer.experts[i].prec, i, layer.d_model, layer.d_ff, False)
                                                  for i, e in enumerate(self.host_experts)])
        self.slot_bytes = int(lib().moe_swap_slot_bytes(ctypes.byref(layer.c)))
        self.space = torch.empty(max(1, n_slots * self.slot_bytes), dtype=torch.uint8, device="cuda")
        self.host_idx = torch.empty(n_tokens * layer.top_k, dtype=torch.int32).pin_memory()
        self.copy_stream = torch.cuda.Stream()
        self.copied, self.computed = torch.cuda.Event(), torch.cuda.Event()
        # torch creates the underlying hipEvent_t lazily, on the first record
        self.copied.record(self.copy_stream)
        self.computed.record(self.copy_stream)
        self.c = CSwap(self._arr, _ptr(self.space), self.slot_bytes, n_slots, self.host_idx.data_ptr(),
                       self.copy_stream.cuda_stream, self.copied.cuda_event, self.computed.cuda_event)


def moe_layer_forward_swap(layer: Layer, swap: Swap, x, out, ws, topk_idx_out=None, topk_gate_out=None) -> int:
    """Returns the number of experts copied in by this call."""
    missed = ctypes.c_int32(0)
    _check(lib().moe_layer_forward_swap(ctypes.byref(layer.c), ctypes.byref(swap.c), _ptr(x), x.shape[0], _ptr(out),
                                        _ptr(topk_idx_out), _ptr(topk_gate_out), _ptr(ws), ws.numel(), _stream(),
                                        ctypes.byref(missed)))
    return missed.value


class Chain:
    """Host arrays for moe_chain_forward, built once."""

    def __init__(self, layers: Sequence[Layer], rms_gains: Sequence):
        self.layers, self.rms_gains = list(layers), list(rms_gains)
        self.c_layers = (CLayer * len(self.layers))(*[l.c for l in self.layers])
        self.c_gains = (ctypes.c_void_p * len(self.layers))(*[_ptr(g) for g in self.rms_gains])


def moe_chain_forward(chain: Chain, eps: float, h, ws, topk_idx_out=None) -> None:
    _check(lib().moe_chain_forward(chain.c_layers, chain.c_gains, len(chain.layers), eps, _ptr(h), h.shape[0],
                                   _ptr(topk_idx_out), _ptr(ws), ws.numel(), _stream()))


def moe_dequant_int4(m: Mat, out: int, inn: int, w_fp16) -> None:
    cm = m.c()
    _check(lib().moe_dequant_int4(ctypes.byref(cm), out, inn, _ptr(w_fp16), _stream()))


def moe_quantize_int4(w_fp16, packed, scale, zero) -> None:
    out, inn = w_fp16.shape
    _check(lib().moe_quantize_int4(_ptr(w_fp16), out, inn, _ptr(packed), _ptr(scale), _ptr(zero), _stream()))


def moe_dequant_int8(m: Mat, out: int, inn: int, w_fp16) -> None:
    cm = m.c()
    _check(lib().moe_dequant_int8(ctypes.byref(cm), out, inn, _ptr(w_fp16), _stream()))


def moe_quantize_int8(w_fp16, codes, scale, zero) -> None:
    out, inn = w_fp16.shape
    _check(lib().moe_quantize_int8(_ptr(w_fp16), out, inn, _ptr(codes), _ptr(scale), _ptr(zero), _stream()))


# ---------------------------------------------------------------- 8-bit floating point and the training of the gate
#
# Shapes, types and places of the tensors are looked at before a call (MoeError with MOE_EINVAL or MOE_ESHAPE): the kernels read and write what they
# are told to.  Tensors have to be contiguous and on the current device.

# Types of tensors, filled in by _device(): f16, f32, i32, e4m3 codes, masks
_F16 = _F32 = _I32 = _CODES = _MASK = _BYTES = ()


def _device() -> int:
    """The current GPU, on which the tensors of a call have to be (-1: there is none)."""
    global _F16, _F32, _I32, _CODES, _MASK, _BYTES
    import torch
    if not _F16:
        _F32, _I32, _CODES = (torch.float32,), (torch.int32,), (torch.uint8, torch.float8_e4m3fn)
        _MASK, _BYTES, _F16 = (torch.uint8, torch.bool), (torch.uint8,), (torch.float16,)
    return torch.cuda.current_device() if torch.cuda.is_initialized() or torch.cuda.is_available() else -1


def _stream_on(dev: int) -> int:
    """The current stream's handle, a small part of the time that torch.cuda.current_stream() takes (2.9 us a call)."""
    import torch
    return torch._C._cuda_getCurrentRawStream(dev)


def _need(t, what: str, dtypes, shape, dev: int) -> int:
    """Pointer of tensor ``t``, which has to be contiguous, of one of ``dtypes`` and of ``shape``, on GPU ``dev``."""
    try:
        if t.dtype in dtypes and t.shape == shape and t.is_contiguous() and t.get_device() == dev and dev >= 0:
            return t.data_ptr()
    except AttributeError:
        raise MoeError(MOE_EINVAL, f"{what}: a tensor is needed") from None
    if t.dtype not in dtypes or not t.is_contiguous():
        raise MoeError(MOE_EINVAL, f"{what}: {t.dtype}, strides {t.stride()}: contiguous {dtypes} is needed")
    if t.shape != shape:
        raise MoeError(MOE_ESHAPE, f"{what}: {tuple(t.shape)}, {tuple(shape)} is needed")
    raise MoeError(MOE_EINVAL, f"{what}: on {t.device}, which is not the current GPU")


def _rows_cols(t, what: str):
    if getattr(t, "ndim", 0) != 2:
        raise MoeError(MOE_ESHAPE, f"{what}: two dimensions are needed")
    return t.shape


def _blocks(n: int) -> int:
    return (n + FP8_BLOCK - 1) // FP8_BLOCK


def _need_fp8(m: Mat, what: str, dev: int) -> CMat:
    """C descriptor of an e4m3 matrix whose tensors fit each other."""
    out, inn = _rows_cols(m.data, what)
    return CMat(_need(m.data, what, _CODES, (out, inn), dev), _need(m.scale, "scale of " + what, _F32, (_blocks(out), _blocks(inn)), dev), None)


def _out_type(t, what: str) -> int:
    if t.dtype in _F32:
        return OUT_F32
    if t.dtype in _F16:
        return OUT_F16
    raise MoeError(MOE_EINVAL, f"{what}: {t.dtype}: float32 or float16 is needed")


def moe_quantize_fp8(w_fp16, codes, scale) -> None:
    dev = _device()
    out, inn = _rows_cols(w_fp16, "w_fp16")
    _check(lib().moe_quantize_fp8(_need(w_fp16, "w_fp16", _F16, (out, inn), dev), out, inn, _need(codes, "codes", _CODES, (out, inn), dev),
                                  _need(scale, "scale", _F32, (_blocks(out), _blocks(inn)), dev), _stream_on(dev)))


def moe_dequant_fp8(m: Mat, out: int, inn: int, w_fp16) -> None:
    dev = _device()
    cm = _need_fp8(m, "m", dev)
    if m.data.shape != (out, inn):
        raise MoeError(MOE_ESHAPE, f"m: {tuple(m.data.shape)}, {(out, inn)} is needed")
    _check(lib().moe_dequant_fp8(ctypes.byref(cm), out, inn, _need(w_fp16, "w_fp16", _F16, (out, inn), dev), _stream_on(dev)))


def moe_quantize_fp8_rows(x, codes, scale) -> None:
    dev = _device()
    n, inn = _rows_cols(x, "x")
    _check(lib().moe_quantize_fp8_rows(_need(x, "x", _F16, (n, inn), dev), n, inn, _need(codes, "codes", _CODES, (n, inn), dev),
                                       _need(scale, "scale", _F32, (_blocks(inn), n), dev), _stream_on(dev)))


def moe_transpose_fp8(m: Mat, codes_t, scale_t) -> None:
    dev = _device()
    cm = _need_fp8(m, "m", dev)
    out, inn = m.data.shape
    _check(lib().moe_transpose_fp8(ctypes.byref(cm), out, inn, _need(codes_t, "codes_t", _CODES, (inn, out), dev),
                                   _need(scale_t, "scale_t", _F32, (_blocks(inn), _blocks(out)), dev), _stream_on(dev)))


def moe_matmul_fp8(w: Mat, x_codes, x_scale, y) -> None:
    """y = x W^T: ``x_codes`` [n,in] and ``x_scale`` [ceil(in/128),n] of moe_quantize_fp8_rows, ``y`` [n,out] float32 or float16."""
    dev = _device()
    cm = _need_fp8(w, "w", dev)
    out, inn = w.data.shape
    n = _rows_cols(x_codes, "x_codes")[0]
    _check(lib().moe_matmul_fp8(cm, out, inn, _need(x_codes, "x_codes", _CODES, (n, inn), dev),
                                _need(x_scale, "x_scale", _F32, (_blocks(inn), n), dev), n, _need(y, "y", _F32 + _F16, (n, out), dev),
                                _out_type(y, "y"), _stream_on(dev)))


class MatGroup:
    """Host array of e4m3 matrices of one shape for moe_matmul_fp8_grouped, built once; keeps their tensors alive."""

    def __init__(self, mats: Sequence[Mat]):
        self.mats, dev = list(mats), _device()
        if not 1 <= len(self.mats) <= MAX_EXPERTS:
            raise MoeError(MOE_ESHAPE, f"{len(self.mats)} matrices, 1 to {MAX_EXPERTS} are possible")
        self.c = (CMat * len(self.mats))(*[_need_fp8(m, f"matrix {i}", dev) for i, m in enumerate(self.mats)])
        self.shape, self.device = tuple(self.mats[0].data.shape), dev
        for i, m in enumerate(self.mats):
            if m.data.shape != self.shape:
                raise MoeError(MOE_ESHAPE, f"matrix {i}: {tuple(m.data.shape)}, {self.shape} is needed")


def moe_matmul_fp8_grouped(group: MatGroup, x_codes, x_scale, offsets, perm, top_k: int, y) -> None:
    """``perm`` None: rows of x in order."""
    dev = _device()
    if group.device != dev:
        raise MoeError(MOE_EINVAL, f"matrices on GPU {group.device}, the current one is {dev}")
    (out, inn), E = group.shape, len(group.mats)
    n, P = _rows_cols(x_codes, "x_codes")[0], _rows_cols(y, "y")[0]
    _check(lib().moe_matmul_fp8_grouped(group.c, E, out, inn, _need(x_codes, "x_codes", _CODES, (n, inn), dev),
                                        _need(x_scale, "x_scale", _F32, (_blocks(inn), n), dev), n,
                                        _need(offsets, "offsets", _I32, (E + 1,), dev),
                                        None if perm is None else _need(perm, "perm", _I32, (P,), dev), top_k, P,
                                        _need(y, "y", _F32 + _F16, (P, out), dev), _out_type(y, "y"), _stream_on(dev)))


def moe_route_logits(layer: Layer, x, logits, topk_idx, topk_gate) -> None:
    dev = _device()
    T, E, k = _rows_cols(x, "x")[0], layer.n_experts, layer.top_k
    _need(layer.w_gate, "w_gate", _F16, (E, layer.d_model), dev)
    _check(lib().moe_route_logits(layer.c, _need(x, "x", _F16, (T, layer.d_model), dev), T, _need(logits, "logits", _F32, (T, E), dev),
                                  _need(topk_idx, "topk_idx", _I32, (T, k), dev), _need(topk_gate, "topk_gate", _F32, (T, k), dev),
                                  _stream_on(dev)))


def gate_workspace_bytes(layer: Layer, n_tokens: int) -> int:
    return int(lib().moe_gate_workspace_bytes(ctypes.byref(layer.c), n_tokens))


def alloc_gate_workspace(layer: Layer, n_tokens: int):
    import torch
    n = gate_workspace_bytes(layer, n_tokens)
    if n == 0:
        raise MoeError(MOE_EINVAL, "moe_gate_workspace_bytes rejected the arguments")
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def moe_balance_loss(layer: Layer, logits, topk_idx, counts, mean_prob, loss, ws, valid=None) -> None:
    dev = _device()
    T, E, k = _rows_cols(logits, "logits")[0], layer.n_experts, layer.top_k
    _check(lib().moe_balance_loss(layer.c, _need(logits, "logits", _F32, (T, E), dev), _need(topk_idx, "topk_idx", _I32, (T, k), dev),
                                  None if valid is None else _need(valid, "valid", _MASK, (T,), dev), T,
                                  _need(counts, "counts", _I32, (E + 1,), dev), _need(mean_prob, "mean_prob", _F32, (E,), dev),
                                  _need(loss, "loss", _F32, (1,), dev), None if ws is None else _need(ws, "ws", _BYTES, ws.shape, dev),
                                  0 if ws is None else ws.numel(), _stream_on(dev)))


def moe_route_backward(layer: Layer, x, logits, topk_idx, ws, valid=None, counts=None, d_gate=None, d_loss=None, d_logits=None,
                       d_x=None, d_w_gate=None, d_bias=None) -> None:
    """The gradients that are not None are written; ``d_x`` float32 or float16."""
    dev = _device()
    T, E, k, d = _rows_cols(logits, "logits")[0], layer.n_experts, layer.top_k, layer.d_model
    if d_x is not None:
        _need(layer.w_gate, "w_gate", _F16, (E, d), dev)
    _check(lib().moe_route_backward(
        layer.c, None if x is None else _need(x, "x", _F16, (T, d), dev), _need(logits, "logits", _F32, (T, E), dev),
        _need(topk_idx, "topk_idx", _I32, (T, k), dev), None if valid is None else _need(valid, "valid", _MASK, (T,), dev), T,
        None if counts is None else _need(counts, "counts", _I32, (E + 1,), dev),
        None if d_gate is None else _need(d_gate, "d_gate", _F32, (T, k), dev),
        None if d_loss is None else _need(d_loss, "d_loss", _F32, (1,), dev),
        None if d_logits is None else _need(d_logits, "d_logits", _F32, (T, E), dev),
        None if d_x is None else _need(d_x, "d_x", _F32 + _F16, (T, d), dev), OUT_F32 if d_x is None else _out_type(d_x, "d_x"),
        None if d_w_gate is None else _need(d_w_gate, "d_w_gate", _F32, (E, d), dev),
        None if d_bias is None else _need(d_bias, "d_bias", _F32, (E,), dev),
        None if ws is None else _need(ws, "ws", _BYTES, ws.shape, dev), 0 if ws is None else ws.numel(), _stream_on(dev)))


# ---------------------------------------------------------------- training the experts

def experts_workspace_bytes(layer: Layer, n_tokens: int) -> int:
    return int(lib().moe_experts_workspace_bytes(layer.c, n_tokens))


def alloc_experts_workspace(layer: Layer, n_tokens: int):
    import torch
    n = experts_workspace_bytes(layer, n_tokens)
    if n == 0:
        raise MoeError(MOE_ESHAPE, "moe_experts_workspace_bytes rejected the arguments: " + lib().moe_last_error().decode())
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def _need_experts(layer: Layer, dev: int) -> None:
    """The matrices are 16-bit ones of the layer's shape on the current GPU.  (Looked at once per layer and GPU: a Layer keeps its experts.)"""
    if getattr(layer, "_trained_on", None) == dev:
        return
    d, f = layer.d_model, layer.d_ff
    for i, e in enumerate(layer.experts):
        if e.prec != PREC_FP16:
            raise MoeError(MOE_EINVAL, f"expert {i} is not held in 16 bits")
        if not e.resident or e.w1 is None or e.w3 is None or e.w2 is None:
            raise MoeError(MOE_ENOTRESIDENT, f"expert {i} is not resident")
        for m, name, shape in ((e.w1, "w1", (f, d)), (e.w3, "w3", (f, d)), (e.w2, "w2", (d, f))):
            _need(m.data, f"expert {i}, {name}", _F16, shape, dev)
    layer._trained_on = dev


def _grouping(layer: Layer, T: int, topk_gate, offsets, perm, dev: int):
    E, k = layer.n_experts, layer.top_k
    return (None if topk_gate is None else _need(topk_gate, "topk_gate", _F32, (T, k), dev),
            None if offsets is None else _need(offsets, "offsets", _I32, (E + 1,), dev),
            None if perm is None else _need(perm, "perm", _I32, (T * k,), dev))


def moe_experts_forward(layer: Layer, x, topk_gate, offsets, perm, a, u, out, ws) -> None:
    """``topk_gate`` None: gates of 1; ``offsets`` None: one expert has all rows; ``perm`` None: row r is pair r."""
    dev = _device()
    T, d, f = _rows_cols(x, "x")[0], layer.d_model, layer.d_ff
    _need_experts(layer, dev)
    kept = (T * layer.top_k, f)
    _check(lib().moe_experts_forward(layer.c, _need(x, "x", _F16, (T, d), dev), T, *_grouping(layer, T, topk_gate, offsets, perm, dev),
                                     _need(a, "a", _F16, kept, dev), _need(u, "u", _F16, kept, dev), _need(out, "out", _F16, (T, d), dev),
                                     None if ws is None else _need(ws, "ws", _BYTES, ws.shape, dev), 0 if ws is None else ws.numel(), _stream_on(dev)))


class ExpertGrads:
    """Host array of the gradients of a block's matrices for moe_experts_backward, built once; keeps their tensors alive.  One (w1, w3, w2) per expert, all
    float32 or all float16; None is not asked for."""

    def __init__(self, grads: Sequence):
        self.grads, dev = [tuple(g) if g is not None else (None, None, None) for g in grads], _device()
        if not 1 <= len(self.grads) <= MAX_EXPERTS:
            raise MoeError(MOE_ESHAPE, f"gradients of {len(self.grads)} experts, 1 to {MAX_EXPERTS} are possible")
        self.device, self.type, self.shape, rows = dev, None, None, []
        for i, g in enumerate(self.grads):
            if len(g) != 3:
                raise MoeError(MOE_EINVAL, f"expert {i}: three gradients are needed")
            ptrs = []
            for t, name in zip(g, ("w1", "w3", "w2")):
                if t is None:
                    ptrs.append(None)
                    continue
                shape = tuple(_rows_cols(t, f"expert {i}, {name}"))
                as_w1 = shape[::-1] if name == "w2" else shape
                if self.type is None:
                    self.type, self.shape = t.dtype, as_w1
                    _out_type(t, f"expert {i}, {name}")
                if as_w1 != self.shape:
                    raise MoeError(MOE_ESHAPE, f"expert {i}, {name}: {shape}")
                ptrs.append(_need(t, f"expert {i}, {name}", (self.type,), shape, dev))
            rows.append(CExpertGrads(*ptrs))
        self.c = (CExpertGrads * len(rows))(*rows)


def moe_experts_backward(layer: Layer, x, topk_gate, offsets, perm, a, u, d_out, ws, d_x=None, d_gate=None, d_w: Optional[ExpertGrads] = None,
                         accumulate: bool = False) -> None:
    """The gradients that are not None are written; ``d_x`` float32 or float16."""
    dev = _device()
    T, d, f, E, k = _rows_cols(x, "x")[0], layer.d_model, layer.d_ff, layer.n_experts, layer.top_k
    _need_experts(layer, dev)
    kept = (T * k, f)
    if d_w is not None:
        if d_w.device != dev:
            raise MoeError(MOE_EINVAL, f"gradients on GPU {d_w.device}, the current one is {dev}")
        if len(d_w.grads) != E or d_w.shape not in (None, (f, d)):
            raise MoeError(MOE_ESHAPE, f"gradients of {len(d_w.grads)} experts of {d_w.shape}, {E} of {(f, d)} are needed")
    _check(lib().moe_experts_backward(
        layer.c, _need(x, "x", _F16, (T, d), dev), T, *_grouping(layer, T, topk_gate, offsets, perm, dev), _need(a, "a", _F16, kept, dev),
        _need(u, "u", _F16, kept, dev), _need(d_out, "d_out", _F16, (T, d), dev),
        None if d_x is None else _need(d_x, "d_x", _F32 + _F16, (T, d), dev), OUT_F32 if d_x is None else _out_type(d_x, "d_x"),
        None if d_gate is None else _need(d_gate, "d_gate", _F32, (T, k), dev), None if d_w is None else d_w.c,
        OUT_F16 if d_w is not None and d_w.type in _F16 else OUT_F32, int(accumulate),
        None if ws is None else _need(ws, "ws", _BYTES, ws.shape, dev), 0 if ws is None else ws.numel(), _stream_on(dev)))


class GradList:
    """Host array of gradients for moe_clip_gradients, built once; keeps their tensors alive.  ``outs`` None: clipped in place."""

    def __init__(self, grads: Sequence, outs: Optional[Sequence] = None):
        self.grads, dev = list(grads), _device()
        self.outs = self.grads if outs is None else list(outs)
        if len(self.grads) > MAX_GRADS or len(self.outs) != len(self.grads):
            raise MoeError(MOE_ESHAPE, f"{len(self.grads)} gradients, {len(self.outs)} outs: as many are needed, at most {MAX_GRADS}")
        self.device = dev
        for i, g in enumerate(self.grads):
            if not hasattr(g, "shape"):
                raise MoeError(MOE_EINVAL, f"gradient {i}: a tensor is needed")
        self.c = (CGrad * max(1, len(self.grads)))(*[
            CGrad(_need(g, f"gradient {i}", _F32 + _F16, g.shape, dev), _need(o, f"out {i}", _F32 + _F16, g.shape, dev), g.numel(),
                  _out_type(g, f"gradient {i}"), _out_type(o, f"out {i}")) for i, (g, o) in enumerate(zip(self.grads, self.outs))])


def alloc_clip_workspace(n_tensors: int):
    import torch
    n = int(lib().moe_clip_workspace_bytes(n_tensors))
    if n == 0:
        raise MoeError(MOE_ESHAPE, "moe_clip_workspace_bytes rejected the argument")
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def moe_clip_gradients(grads: GradList, max_norm: float, norm, ws, unscale: float = 1.0) -> None:
    dev = _device()
    if grads.device != dev:
        raise MoeError(MOE_EINVAL, f"gradients on GPU {grads.device}, the current one is {dev}")
    _check(lib().moe_clip_gradients(grads.c, len(grads.grads), max_norm, unscale, _need(norm, "norm", _F32, (1,), dev),
                                    None if ws is None else _need(ws, "ws", _BYTES, ws.shape, dev), 0 if ws is None else ws.numel(), _stream_on(dev)))


def moe_synth_fill_f16(dst, first: int, seed: int, stream_id: int, scale: float, kind: int) -> None:
    _check(lib().moe_synth_fill_f16(_ptr(dst), dst.numel(), first, seed, stream_id, scale, kind, _stream()))


def moe_read_status(ws) -> int:
    """Status bits of the last call on workspace ``ws`` (None: of the last moe_layer_forward_static call)."""
    v = ctypes.c_int(0)
    _check(lib().moe_read_status(_ptr(ws), _stream(), ctypes.byref(v)))
    return v.value


KERNEL_ROUTE, KERNEL_PERMUTE, KERNEL_UP, KERNEL_DOWN, KERNEL_COMBINE, KERNEL_STREAM_READ = range(6)


def moe_trace_kernel(kernel: int, start_event: Optional[int], stop_event: Optional[int]) -> None:
    """Arms a one-shot event bracket around the next launch of ``kernel``; (None, None) drops an unused one."""
    _check(lib().moe_trace_kernel(kernel, start_event, stop_event))


def moe_stream_read(src, nbytes: int, sink) -> None:
    _check(lib().moe_stream_read(_ptr(src), nbytes, _ptr(sink), _stream()))


def moe_plan(mem_gpu: int, size_non_expert: int, size_e16: int, size_e4: int, num_experts: int, preference: int,
             num_e4: int = 0, seed: int = 0, swap_bytes: int = 0):
    """Returns (CPlanResult, quantized list, resident list); host-only."""
    req = CPlanRequest(mem_gpu, size_non_expert, size_e16, size_e4, swap_bytes, seed, num_experts, preference, num_e4)
    res = CPlanResult()
    q = (ctypes.c_uint8 * max(num_experts, 1))()
    r = (ctypes.c_uint8 * max(num_experts, 1))()
    rc = lib().moe_plan(ctypes.byref(req), ctypes.byref(res), q, r)
    if rc != MOE_OK:
        raise MoeError(rc, "moe_plan rejected the request")
    return res, list(q)[:num_experts], list(r)[:num_experts]


def moe_version() -> int:
    return int(lib().moe_version())


# ---------------------------------------------------------------- conveniences built only from the calls above

def quantize_mat(w_fp16) -> Mat:
    """Device-side 16-bit -> 4-bit switch of one matrix (moe_quantize_int4)."""
    import torch
    out, inn = w_fp16.shape
    packed = torch.empty((out, inn // 2), dtype=torch.uint8, device=w_fp16.device)
    scale = torch.empty((out, inn // GROUP), dtype=torch.float16, device=w_fp16.device)
    zero = torch.empty((out, inn // GROUP), dtype=torch.float16, device=w_fp16.device)
    moe_quantize_int4(w_fp16, packed, scale, zero)
    return Mat(packed, scale, zero)


def quantize_mat8(w_fp16) -> Mat:
    """Device-side 16-bit -> 8-bit switch of one matrix (moe_quantize_int8)."""
    import torch
    out, inn = w_fp16.shape
    codes = torch.empty((out, inn), dtype=torch.uint8, device=w_fp16.device)
    scale = torch.empty((out, inn // GROUP), dtype=torch.float16, device=w_fp16.device)
    zero = torch.empty((out, inn // GROUP), dtype=torch.float16, device=w_fp16.device)
    moe_quantize_int8(w_fp16, codes, scale, zero)
    return Mat(codes, scale, zero)


def quantize_mat_fp8(w_fp16) -> Mat:
    """Device-side 16-bit -> e4m3 switch of one matrix (moe_quantize_fp8)."""
    import torch
    out, inn = w_fp16.shape
    codes = torch.empty((out, inn), dtype=torch.uint8, device=w_fp16.device)
    scale = torch.empty((_blocks(out), _blocks(inn)), dtype=torch.float32, device=w_fp16.device)
    moe_quantize_fp8(w_fp16, codes, scale)
    return Mat(codes, scale)


def transpose_mat_fp8(m: Mat) -> Mat:
    """The transposed e4m3 matrix (moe_transpose_fp8)."""
    import torch
    out, inn = m.data.shape
    codes = torch.empty((inn, out), dtype=torch.uint8, device=m.data.device)
    scale = torch.empty((_blocks(inn), _blocks(out)), dtype=torch.float32, device=m.data.device)
    moe_transpose_fp8(m, codes, scale)
    return Mat(codes, scale)

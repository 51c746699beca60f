"""Thin ctypes binding of the C ABI in include/osc.h (argument marshalling only).

Every function here has the name of the C entry point it calls.  torch is used
for device memory and streams; all arithmetic happens in the CUDA library.
Importing this module loads `libosc_b200.so` from the package directory and
raises if it is missing: there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libosc_b200.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} not found: build it with `python -c 'import __graft_entry__ as g; g.build()'` "
                      "(nvcc, sm_100a). The OSC path has no CPU fallback.")
_lib = C.CDLL(LIB_PATH)

OSC_OK = 0
STATUS = {0: "OSC_OK", -1: "OSC_ERR_INVALID_ARG", -2: "OSC_ERR_SHAPE", -3: "OSC_ERR_LUT", -4: "OSC_ERR_ALIGN",
          -5: "OSC_ERR_WORKSPACE", -6: "OSC_ERR_ARCH", -7: "OSC_ERR_CUDA", -8: "OSC_ERR_TIMEOUT"}


class OscError(RuntimeError):
    def __init__(self, status: int, detail: str):
        super().__init__(f"{STATUS.get(status, status)}: {detail}")
        self.status = status


class WeightSizes(C.Structure):
    _fields_ = [("K_o", C.c_int32), ("K_o_pad", C.c_int32), ("wq_bytes", C.c_size_t), ("sfw_bytes", C.c_size_t),
                ("wo_bytes", C.c_size_t), ("meta_bytes", C.c_size_t)]


class ActSizes(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("xq_bytes", "sfa_bytes", "xo_bytes", "sched_bytes", "xq_offset",
                                          "sfa_offset", "xo_offset", "sched_offset", "workspace_bytes")]


class Fp8ActSizes(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("x8_bytes", "sx_bytes", "sched_bytes", "x8_offset", "sx_offset",
                                          "sched_offset", "workspace_bytes")]


class DynActSizes(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("xq_bytes", "sfa_bytes", "xo_bytes", "idx_bytes", "val_bytes", "xq_offset",
                                          "sfa_offset", "xo_offset", "idx_offset", "val_offset", "workspace_bytes")]


class Mxfp8WeightSizes(C.Structure):
    _fields_ = [("w8_bytes", C.c_size_t), ("sfw_bytes", C.c_size_t)]


class Mxfp8ActSizes(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("x8_bytes", "sfa_bytes", "sched_bytes", "x8_offset", "sfa_offset",
                                          "sched_offset", "workspace_bytes")]


class KvCacheStruct(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_heads", C.c_int32),
                ("head_dim", C.c_int32), ("page_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class RopeStruct(C.Structure):
    _fields_ = [("inv_freq", C.c_void_p), ("axis", C.c_void_p), ("rot_dim", C.c_int32), ("axes", C.c_int32),
                ("interleaved", C.c_int32), ("scale", C.c_float)]


_vp, _i, _i64, _sz = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
_SIGS = {
    "osc_status_string": (C.c_char_p, [_i]),
    "osc_last_error": (C.c_char_p, []),
    "osc_sync_check": (_i, [_vp]),
    "osc_weight_sizes": (_i, [_i, _i, _i, _vp, _i, C.POINTER(WeightSizes)]),
    "osc_prepare_weights": (_i, [_vp, _i, _i, _i64, _vp, _i, _vp, _vp, _vp, _vp, _vp, C.POINTER(_vp)]),
    "osc_prepare_weights_grouped": (_i, [_vp, _i, _i, _i, _vp, _i, _vp, _vp, _vp, _vp, _vp, C.POINTER(_vp)]),
    "osc_weights_destroy": (_i, [_vp]),
    "osc_act_sizes": (_i, [_vp, _i, C.POINTER(ActSizes)]),
    "osc_quantize_extract": (_i, [_vp, _vp, _i, _i64, _vp, _vp, _vp, _vp]),
    "osc_gemm_dual": (_i, [_vp, _vp, _vp, _vp, _i, _vp, _i64, _vp]),
    "osc_linear": (_i, [_vp, _vp, _i, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_linear_static": (_i, [_vp, _vp, _i, _i64, _vp, _i64, _vp]),
    "osc_linear_grouped": (_i, [_vp, _vp, _vp, _i, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_gather_workspace_bytes": (_i, [_vp, _i, _i, C.POINTER(_sz)]),
    "osc_linear_grouped_gather": (_i, [_vp, _vp, _i, _i64, _vp, _vp, _i, _vp, _i64, _vp, _sz, _vp]),
    "osc_rmsnorm_linear_grouped_gather": (_i, [_vp, _vp, _i, _i64, _vp, C.c_float, _vp, _vp, _i, _vp, _i64, _vp, _sz, _vp]),
    "osc_swiglu_fp8_linear_grouped": (_i, [_vp, _vp, _vp, _i, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_add_rmsnorm": (_i, [_vp, _vp, _i, _i, _i64, _i64, _vp, C.c_float, _vp, _i64, _vp, _i64, _vp]),
    "osc_add_rmsnorm_quantize_extract": (_i, [_vp, _vp, _vp, _i, _i64, _i64, _vp, C.c_float, _vp, _i64, _vp, _vp, _vp, _vp]),
    "osc_add_rmsnorm_linear": (_i, [_vp, _vp, _vp, _i, _i64, _i64, _vp, C.c_float, _vp, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_rmsnorm": (_i, [_vp, _i, _i, _i64, _vp, C.c_float, _vp, _i64, _vp]),
    "osc_swiglu": (_i, [_vp, _i, _i, _i64, _vp, _i64, _vp]),
    "osc_swiglu_fp8_quantize": (_i, [_vp, _i, _i, _i64, _vp, _vp, _vp]),
    "osc_swiglu_fp8_linear": (_i, [_vp, _vp, _i, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_rmsnorm_quantize_extract": (_i, [_vp, _vp, _i, _i64, _vp, C.c_float, _vp, _vp, _vp, _vp]),
    "osc_rmsnorm_linear": (_i, [_vp, _vp, _i, _i64, _vp, C.c_float, _vp, _i64, _vp, _sz, _vp]),
    "osc_profile_scratch_bytes": (_i, [_i, C.POINTER(_sz)]),
    "osc_profile_lut": (_i, [_vp, _i, _i, _i64, C.c_float, _vp, _sz, _vp, _vp, _vp, _vp, _vp]),
    "osc_fp8_prepare_weights": (_i, [_vp, _i, _i, _i64, _vp, _vp, _vp, C.POINTER(_vp)]),
    "osc_fp8_prepare_weights_grouped": (_i, [_vp, _i, _i, _i, _vp, _vp, _vp, C.POINTER(_vp)]),
    "osc_fp8_weights_destroy": (_i, [_vp]),
    "osc_fp8_act_sizes": (_i, [_vp, _i, C.POINTER(Fp8ActSizes)]),
    "osc_fp8_quantize": (_i, [_vp, _i, _i, _i64, _vp, _vp, _vp]),
    "osc_fp8_gemm": (_i, [_vp, _vp, _vp, _i, _vp, _i64, _vp]),
    "osc_fp8_linear": (_i, [_vp, _vp, _i, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_fp8_linear_grouped": (_i, [_vp, _vp, _vp, _i, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_dyn_weight_sizes": (_i, [_i, _i, C.POINTER(WeightSizes)]),
    "osc_dyn_prepare_weights": (_i, [_vp, _i, _i, _i64, _vp, _vp, _vp, _vp, _vp, C.POINTER(_vp)]),
    "osc_dyn_act_sizes": (_i, [_vp, _i, C.POINTER(DynActSizes)]),
    "osc_dyn_quantize_extract": (_i, [_vp, _vp, _i, _i64, _vp, _vp, _vp, _vp, _vp, _vp]),
    "osc_dyn_linear": (_i, [_vp, _vp, _i, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_nvfp4_weight_sizes": (_i, [_i, _i, _vp, _i, C.POINTER(WeightSizes)]),
    "osc_nvfp4_prepare_weights": (_i, [_vp, _i, _i, _i64, _vp, _i, _i, _vp, _vp, _vp, _vp, _vp, C.POINTER(_vp)]),
    "osc_nvfp4_weight_sizes_grouped": (_i, [_i, _i, _i, _vp, _i, C.POINTER(WeightSizes)]),
    "osc_nvfp4_prepare_weights_grouped": (_i, [_vp, _i, _i, _i, _vp, _i, _i, _vp, _vp, _vp, _vp, _vp, C.POINTER(_vp)]),
    "osc_nvfp4_linear_grouped": (_i, [_vp, _vp, _vp, _i, _i64, _i, _vp, _i64, _vp, _sz, _vp]),
    "osc_nvfp4_act_sizes": (_i, [_vp, _i, C.POINTER(ActSizes)]),
    "osc_nvfp4_quantize_extract": (_i, [_vp, _vp, _i, _i64, _i, _vp, _vp, _vp, _vp]),
    "osc_nvfp4_gemm": (_i, [_vp, _vp, _vp, _vp, _i, _i, _vp, _i64, _vp]),
    "osc_nvfp4_linear": (_i, [_vp, _vp, _i, _i64, _i, _vp, _i64, _vp, _sz, _vp]),
    "osc_gate_up_weight_sizes": (_i, [_i, _i, _vp, _i, C.POINTER(WeightSizes)]),
    "osc_prepare_weights_gate_up": (_i, [_vp, _i, _i, _i64, _vp, _i, _vp, _vp, _vp, _vp, _vp, C.POINTER(_vp)]),
    "osc_linear_swiglu_workspace_bytes": (_i, [_vp, _i, C.POINTER(_sz)]),
    "osc_linear_swiglu": (_i, [_vp, _vp, _i, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_rmsnorm_linear_swiglu": (_i, [_vp, _vp, _i, _i64, _vp, C.c_float, _vp, _i64, _vp, _sz, _vp]),
    "osc_gate_up_weight_sizes_grouped": (_i, [_i, _i, _i, _vp, _i, C.POINTER(WeightSizes)]),
    "osc_prepare_weights_gate_up_grouped": (_i, [_vp, _i, _i, _i, _vp, _i, _vp, _vp, _vp, _vp, _vp, C.POINTER(_vp)]),
    "osc_linear_swiglu_grouped": (_i, [_vp, _vp, _vp, _i, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_swiglu_gather_workspace_bytes": (_i, [_vp, _i, _i, C.POINTER(_sz)]),
    "osc_linear_swiglu_grouped_gather": (_i, [_vp, _vp, _i, _i64, _vp, _vp, _i, _vp, _i64, _vp, _sz, _vp]),
    "osc_rmsnorm_linear_swiglu_grouped_gather": (_i, [_vp, _vp, _i, _i64, _vp, C.c_float, _vp, _vp, _i, _vp, _i64, _vp, _sz, _vp]),
    "osc_nvfp4_rmsnorm_quantize_extract": (_i, [_vp, _vp, _i, _i64, _vp, C.c_float, _i, _vp, _vp, _vp, _vp]),
    "osc_nvfp4_rmsnorm_linear": (_i, [_vp, _vp, _i, _i64, _vp, C.c_float, _i, _vp, _i64, _vp, _sz, _vp]),
    "osc_nvfp4_gather_workspace_bytes": (_i, [_vp, _i, _i, C.POINTER(_sz)]),
    "osc_nvfp4_linear_grouped_gather": (_i, [_vp, _vp, _i, _i64, _vp, _vp, _i, _i, _vp, _i64, _vp, _sz, _vp]),
    "osc_nvfp4_rmsnorm_linear_grouped_gather": (_i, [_vp, _vp, _i, _i64, _vp, C.c_float, _vp, _vp, _i, _i, _vp, _i64, _vp, _sz,
                                                     _vp]),
    "osc_mxfp8_weight_sizes": (_i, [_i, _i, _i, C.POINTER(Mxfp8WeightSizes)]),
    "osc_mxfp8_prepare_weights_grouped": (_i, [_vp, _i, _i, _i, _vp, _vp, _vp, C.POINTER(_vp)]),
    "osc_mxfp8_linear_grouped": (_i, [_vp, _vp, _vp, _i, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_mxfp8_prepare_weights": (_i, [_vp, _i, _i, _i64, _vp, _vp, _vp, C.POINTER(_vp)]),
    "osc_mxfp8_weights_destroy": (_i, [_vp]),
    "osc_mxfp8_act_sizes": (_i, [_vp, _i, C.POINTER(Mxfp8ActSizes)]),
    "osc_mxfp8_quantize": (_i, [_vp, _i, _i, _i64, _vp, _vp, _vp]),
    "osc_mxfp8_gemm": (_i, [_vp, _vp, _vp, _i, _vp, _i64, _vp]),
    "osc_mxfp8_linear": (_i, [_vp, _vp, _i, _i64, _vp, _i64, _vp, _sz, _vp]),
    "osc_kv_slots": (_i, [_vp, _vp, _vp, _i, _i, _vp, _i, _vp, _i, _i64, _i, _vp, _vp, _vp, _vp, _vp, _vp]),
    "osc_qk_norm_rope": (_i, [_vp, _i, _i64, _i, C.POINTER(KvCacheStruct), _vp, _vp, C.c_float, C.POINTER(RopeStruct), _vp, _i64,
                              _vp, _vp, _i64, _vp]),
    "osc_paged_attention_workspace_bytes": (_i, [_i, _i, _i, _i, _i, C.POINTER(_sz)]),
    "osc_paged_attention": (_i, [_vp, _i, _i64, _i, C.POINTER(KvCacheStruct), _i, _vp, _vp, _vp, _i, _i64, _i, _vp, _vp, _vp, _i,
                                 _i64, _i, C.c_float, _vp, _i64, _vp, _vp, _sz, _vp]),
    "osc_tree_mask": (_i, [_vp, _vp, _vp, _i, _i, _vp, _i, _i64, _vp, _vp]),
    "osc_tree_attention": (_i, [_vp, _i, _i64, _i, C.POINTER(KvCacheStruct), _i, _vp, _vp, _vp, _i, _i64, _i, _vp, _vp, _vp, _i,
                                _i64, _vp, _i, _i64, _i, C.c_float, _vp, _i64, _vp, _vp, _sz, _vp]),
    "osc_token_logprobs": (_i, [_vp, _i, _i, _i, _i64, C.c_float, _vp, _i, _i64, _vp, _vp, _vp, _i, _vp, _vp, _vp]),
    "osc_kv_compact": (_i, [_vp, _i, _i, _vp, _vp, _vp, _i, _i64, _vp, _i, _i64, _vp, _vp, _vp]),
    "osc_kv_trim": (_i, [_vp, _vp, _i, _i, _vp, _i, _i64, _vp, _i, _vp, _vp, _vp]),
    "osc_kv_fork": (_i, [_vp, _vp, _i, _vp, _i, _i, _vp, _i, _vp, _i, _i64, _vp, _i, _vp, _vp, _vp, _vp, _vp]),
    "osc_kv_copy_pages": (_i, [_vp, _i, _vp, _vp, _vp, _i, _vp]),
}
for _name, (_res, _args) in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args

EXPORTS = tuple(_SIGS)


def osc_last_error() -> str:
    return _lib.osc_last_error().decode()


def osc_status_string(s: int) -> str:
    return _lib.osc_status_string(s).decode()


def _check(status: int):
    if status != OSC_OK:
        raise OscError(status, osc_last_error())


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        return t.data_ptr() if t.numel() > 0 else None
    return int(t)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream=None):
    """cudaStream_t of `stream`, or of torch's current stream.  Building a torch.cuda.Stream object for the current
    stream costs ~3 us per call, a third of a few-row linear; torch's raw accessor gives the handle directly."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and _raw_device is not None:
        return _raw_stream(_raw_device())
    return torch.cuda.current_stream().cuda_stream


def _lut(lut):
    lut = np.ascontiguousarray(lut, dtype=np.int8)
    if lut.ndim == 1:
        lut = lut.reshape(-1, 1)
    return lut


def osc_sync_check(stream=None):
    _check(_lib.osc_sync_check(_stream(stream)))


def osc_weight_sizes(E: int, N: int, K: int, lut) -> WeightSizes:
    lut = _lut(lut)
    out = WeightSizes()
    _check(_lib.osc_weight_sizes(E, N, K, lut.ctypes.data, lut.shape[1], C.byref(out)))
    return out


class _Handle:
    _destroy = None

    def __init__(self, ptr, keep):
        self.ptr = ptr
        self.keep = keep  # device buffers the handle borrows

    def close(self):
        if self.ptr:
            self._destroy(self.ptr)
            self.ptr = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class OscWeights(_Handle):
    _destroy = staticmethod(_lib.osc_weights_destroy)


class Fp8Weights(_Handle):
    _destroy = staticmethod(_lib.osc_fp8_weights_destroy)


class Mxfp8Weights(_Handle):
    _destroy = staticmethod(_lib.osc_mxfp8_weights_destroy)


def _alloc(nbytes, dev):
    return torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=dev)


def osc_prepare_weights(W: torch.Tensor, lut, stream=None) -> OscWeights:
    """W: cuda bf16 [N, K] (row stride = ldw). Returns a handle owning wq/sfw/wo/meta."""
    N, K = W.shape
    lut = _lut(lut)
    sz = osc_weight_sizes(1, N, K, lut)
    dev = W.device
    bufs = {k: _alloc(getattr(sz, k + "_bytes"), dev) for k in ("wq", "sfw", "wo", "meta")}
    h = _vp()
    _check(_lib.osc_prepare_weights(_ptr(W), N, K, W.stride(0), lut.ctypes.data, lut.shape[1], _ptr(bufs["wq"]),
                                    _ptr(bufs["sfw"]), _ptr(bufs["wo"]) if sz.wo_bytes else None, _ptr(bufs["meta"]),
                                    _stream(stream), C.byref(h)))
    w = OscWeights(h.value, bufs)
    w.E, w.N, w.K, w.K_o, w.K_o_pad, w.sizes = 1, N, K, sz.K_o, sz.K_o_pad, sz
    return w


def osc_prepare_weights_grouped(W: torch.Tensor, lut, stream=None) -> OscWeights:
    """W: cuda bf16 [E, N, K] contiguous."""
    E, N, K = W.shape
    assert W.is_contiguous()
    lut = _lut(lut)
    sz = osc_weight_sizes(E, N, K, lut)
    dev = W.device
    bufs = {k: _alloc(getattr(sz, k + "_bytes"), dev) for k in ("wq", "sfw", "wo", "meta")}
    h = _vp()
    _check(_lib.osc_prepare_weights_grouped(_ptr(W), E, N, K, lut.ctypes.data, lut.shape[1], _ptr(bufs["wq"]),
                                            _ptr(bufs["sfw"]), _ptr(bufs["wo"]) if sz.wo_bytes else None,
                                            _ptr(bufs["meta"]), _stream(stream), C.byref(h)))
    w = OscWeights(h.value, bufs)
    w.E, w.N, w.K, w.K_o, w.K_o_pad, w.sizes = E, N, K, sz.K_o, sz.K_o_pad, sz
    return w


def osc_weights_destroy(w: OscWeights):
    w.close()


def osc_act_sizes(w: OscWeights, M: int) -> ActSizes:
    out = ActSizes()
    _check(_lib.osc_act_sizes(w.ptr, M, C.byref(out)))
    return out


def osc_quantize_extract(w: OscWeights, X: torch.Tensor, xq, sfa, xo, stream=None):
    M = X.shape[0]
    _check(_lib.osc_quantize_extract(w.ptr, _ptr(X), M, X.stride(0) if M else w.K, _ptr(xq), _ptr(sfa),
                                     _ptr(xo) if w.K_o_pad else None, _stream(stream)))


def osc_gemm_dual(w: OscWeights, xq, sfa, xo, M: int, Y: torch.Tensor, stream=None):
    _check(_lib.osc_gemm_dual(w.ptr, _ptr(xq), _ptr(sfa), _ptr(xo) if w.K_o_pad else None, M, _ptr(Y),
                              Y.stride(0) if M else w.N, _stream(stream)))


def osc_linear(w: OscWeights, X: torch.Tensor, Y: torch.Tensor, workspace: torch.Tensor, stream=None):
    M = X.shape[0]
    _check(_lib.osc_linear(w.ptr, _ptr(X), M, X.stride(0) if M else w.K, _ptr(Y), Y.stride(0) if M else w.N,
                           _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_linear_static(w: OscWeights, X: torch.Tensor, Y: torch.Tensor, stream=None):
    """osc_linear for callers that cannot provide a workspace: the scratch is a fixed array inside the
    library (limited size, shared by all calls on a device); nothing is allocated here or in the library."""
    M = X.shape[0]
    _check(_lib.osc_linear_static(w.ptr, _ptr(X), M, X.stride(0) if M else w.K, _ptr(Y), Y.stride(0) if M else w.N,
                                  _stream(stream)))


def osc_gather_workspace_bytes(w: OscWeights, T: int, M_total: int) -> int:
    out = _sz()
    _check(_lib.osc_gather_workspace_bytes(w.ptr, T, M_total, C.byref(out)))
    return int(out.value)


def osc_linear_grouped_gather(w: OscWeights, X: torch.Tensor, row_token: torch.Tensor, off: torch.Tensor, Y: torch.Tensor,
                              workspace: torch.Tensor, stream=None):
    """Grouped linear on X[row_token] without materialising it: tokens quantized once, quantized rows gathered."""
    T, M = X.shape[0], row_token.shape[0]
    _check(_lib.osc_linear_grouped_gather(w.ptr, _ptr(X), T, X.stride(0) if T else w.K, _ptr(row_token), _ptr(off), M,
                                          _ptr(Y), Y.stride(0) if M else w.N, _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_rmsnorm_linear_grouped_gather(w: OscWeights, H: torch.Tensor, gamma: torch.Tensor, eps: float, row_token: torch.Tensor,
                                      off: torch.Tensor, Y: torch.Tensor, workspace: torch.Tensor, stream=None):
    """osc_linear_grouped_gather with the RMSNorm of the residual stream H fused into the quantizer."""
    T, M = H.shape[0], row_token.shape[0]
    _check(_lib.osc_rmsnorm_linear_grouped_gather(w.ptr, _ptr(H), T, H.stride(0) if T else w.K, _ptr(gamma), float(eps),
                                                  _ptr(row_token), _ptr(off), M, _ptr(Y), Y.stride(0) if M else w.N,
                                                  _ptr(workspace), workspace.numel() * workspace.element_size(),
                                                  _stream(stream)))


def osc_rmsnorm(H: torch.Tensor, gamma: torch.Tensor, eps: float, X: torch.Tensor, stream=None):
    """X = bf16(RMSNorm(H) * gamma) (statistic in double, element-wise part in fp32, one rounding to bf16):
    the unfused reference point."""
    M, K = H.shape
    _check(_lib.osc_rmsnorm(_ptr(H), M, K, H.stride(0) if M else K, _ptr(gamma), float(eps), _ptr(X),
                            X.stride(0) if M else K, _stream(stream)))


def osc_add_rmsnorm(H: torch.Tensor, R: torch.Tensor, gamma: torch.Tensor, eps: float, Hout: torch.Tensor, X: torch.Tensor,
                    stream=None):
    """Hout = bf16(H + R), X = RMSNorm(Hout) * gamma: the unfused reference point of the residual form."""
    M, K = H.shape
    _check(_lib.osc_add_rmsnorm(_ptr(H), _ptr(R), M, K, H.stride(0) if M else K, R.stride(0) if M else K, _ptr(gamma),
                                float(eps), _ptr(Hout), Hout.stride(0) if M else K, _ptr(X), X.stride(0) if M else K,
                                _stream(stream)))


def osc_add_rmsnorm_quantize_extract(w: OscWeights, H: torch.Tensor, R: torch.Tensor, gamma: torch.Tensor, eps: float,
                                     Hout: torch.Tensor, xq, sfa, xo, stream=None):
    """Residual update, RMSNorm and Algorithm 2 in one pass: Hout = bf16(H + R) is the only full-width tensor written."""
    M = H.shape[0]
    _check(_lib.osc_add_rmsnorm_quantize_extract(w.ptr, _ptr(H), _ptr(R), M, H.stride(0) if M else w.K,
                                                 R.stride(0) if M else w.K, _ptr(gamma), float(eps), _ptr(Hout),
                                                 Hout.stride(0) if M else w.K, _ptr(xq), _ptr(sfa),
                                                 _ptr(xo) if w.K_o_pad else None, _stream(stream)))


def osc_add_rmsnorm_linear(w: OscWeights, H: torch.Tensor, R: torch.Tensor, gamma: torch.Tensor, eps: float,
                           Hout: torch.Tensor, Y: torch.Tensor, workspace: torch.Tensor, stream=None):
    M = H.shape[0]
    _check(_lib.osc_add_rmsnorm_linear(w.ptr, _ptr(H), _ptr(R), M, H.stride(0) if M else w.K, R.stride(0) if M else w.K,
                                       _ptr(gamma), float(eps), _ptr(Hout), Hout.stride(0) if M else w.K, _ptr(Y),
                                       Y.stride(0) if M else w.N, _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_rmsnorm_quantize_extract(w: OscWeights, H: torch.Tensor, gamma: torch.Tensor, eps: float, xq, sfa, xo, stream=None):
    """RMSNorm fused in front of Algorithm 2: H is read once, the normalized tensor is never written."""
    M = H.shape[0]
    _check(_lib.osc_rmsnorm_quantize_extract(w.ptr, _ptr(H), M, H.stride(0) if M else w.K, _ptr(gamma), float(eps),
                                             _ptr(xq), _ptr(sfa), _ptr(xo) if w.K_o_pad else None, _stream(stream)))


def osc_rmsnorm_linear(w: OscWeights, H: torch.Tensor, gamma: torch.Tensor, eps: float, Y: torch.Tensor,
                       workspace: torch.Tensor, stream=None):
    M = H.shape[0]
    _check(_lib.osc_rmsnorm_linear(w.ptr, _ptr(H), M, H.stride(0) if M else w.K, _ptr(gamma), float(eps), _ptr(Y),
                                   Y.stride(0) if M else w.N, _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_swiglu(GU: torch.Tensor, I: int, H: torch.Tensor, stream=None):
    """H = bf16(silu(GU[:, :I]) * GU[:, I:2I]) in the library's fixed fp32 arithmetic: the unfused reference point."""
    M = GU.shape[0]
    _check(_lib.osc_swiglu(_ptr(GU), M, I, GU.stride(0) if M else 2 * I, _ptr(H), H.stride(0) if M else I, _stream(stream)))


def osc_swiglu_fp8_quantize(GU: torch.Tensor, I: int, x8, sx, stream=None):
    """SwiGLU fused in front of the per-token FP8 quantizer: the activation h is never written."""
    M = GU.shape[0]
    _check(_lib.osc_swiglu_fp8_quantize(_ptr(GU), M, I, GU.stride(0) if M else 2 * I, _ptr(x8), _ptr(sx), _stream(stream)))


def osc_swiglu_fp8_linear(w: "Fp8Weights", GU: torch.Tensor, Y: torch.Tensor, workspace: torch.Tensor, stream=None):
    M = GU.shape[0]
    _check(_lib.osc_swiglu_fp8_linear(w.ptr, _ptr(GU), M, GU.stride(0) if M else 2 * w.K, _ptr(Y),
                                      Y.stride(0) if M else w.N, _ptr(workspace),
                                      workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_swiglu_fp8_linear_grouped(w: "Fp8Weights", GU: torch.Tensor, off: torch.Tensor, Y: torch.Tensor,
                                  workspace: torch.Tensor, stream=None):
    """Grouped FP8 linear on silu(gate) * up of the experts' gate|up rows, the activation never written."""
    M = GU.shape[0]
    _check(_lib.osc_swiglu_fp8_linear_grouped(w.ptr, _ptr(GU), _ptr(off), M, GU.stride(0) if M else 2 * w.K, _ptr(Y),
                                              Y.stride(0) if M else w.N, _ptr(workspace),
                                              workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_linear_grouped(w: OscWeights, X: torch.Tensor, off: torch.Tensor, Y: torch.Tensor, workspace: torch.Tensor,
                       stream=None):
    M = X.shape[0]
    _check(_lib.osc_linear_grouped(w.ptr, _ptr(X), _ptr(off), M, X.stride(0) if M else w.K, _ptr(Y),
                                   Y.stride(0) if M else w.N, _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_profile_scratch_bytes(K: int) -> int:
    out = _sz()
    _check(_lib.osc_profile_scratch_bytes(K, C.byref(out)))
    return int(out.value)


def osc_profile_lut(X: torch.Tensor, alpha: float, scratch, lut, n_hit, n_total, threshold_bits, stream=None):
    """X: cuda bf16 [S, K]; outputs are cuda tensors (int8 [K/32], int32 [K/32] x2, int32/uint32 [1])."""
    S, K = X.shape
    _check(_lib.osc_profile_lut(_ptr(X), S, K, X.stride(0), float(alpha), _ptr(scratch),
                                scratch.numel() * scratch.element_size(), _ptr(lut), _ptr(n_hit), _ptr(n_total),
                                _ptr(threshold_bits), _stream(stream)))


def osc_fp8_prepare_weights(W: torch.Tensor, stream=None) -> Fp8Weights:
    N, K = W.shape
    dev = W.device
    bufs = {"w8": _alloc(N * K, dev), "sw": torch.empty(N, dtype=torch.float32, device=dev)}
    h = _vp()
    _check(_lib.osc_fp8_prepare_weights(_ptr(W), N, K, W.stride(0), _ptr(bufs["w8"]), _ptr(bufs["sw"]),
                                        _stream(stream), C.byref(h)))
    w = Fp8Weights(h.value, bufs)
    w.E, w.N, w.K = 1, N, K
    return w


def osc_fp8_prepare_weights_grouped(W: torch.Tensor, stream=None) -> Fp8Weights:
    E, N, K = W.shape
    assert W.is_contiguous()
    dev = W.device
    bufs = {"w8": _alloc(E * N * K, dev), "sw": torch.empty(E * N, dtype=torch.float32, device=dev)}
    h = _vp()
    _check(_lib.osc_fp8_prepare_weights_grouped(_ptr(W), E, N, K, _ptr(bufs["w8"]), _ptr(bufs["sw"]),
                                                _stream(stream), C.byref(h)))
    w = Fp8Weights(h.value, bufs)
    w.E, w.N, w.K = E, N, K
    return w


def osc_fp8_weights_destroy(w: Fp8Weights):
    w.close()


def osc_fp8_act_sizes(w: Fp8Weights, M: int) -> Fp8ActSizes:
    out = Fp8ActSizes()
    _check(_lib.osc_fp8_act_sizes(w.ptr, M, C.byref(out)))
    return out


def osc_fp8_quantize(X: torch.Tensor, x8, sx, stream=None):
    M, K = X.shape
    _check(_lib.osc_fp8_quantize(_ptr(X), M, K, X.stride(0) if M else K, _ptr(x8), _ptr(sx), _stream(stream)))


def osc_fp8_gemm(w: Fp8Weights, x8, sx, M: int, Y: torch.Tensor, stream=None):
    _check(_lib.osc_fp8_gemm(w.ptr, _ptr(x8), _ptr(sx), M, _ptr(Y), Y.stride(0) if M else w.N, _stream(stream)))


def osc_fp8_linear(w: Fp8Weights, X: torch.Tensor, Y: torch.Tensor, workspace: torch.Tensor, stream=None):
    M = X.shape[0]
    _check(_lib.osc_fp8_linear(w.ptr, _ptr(X), M, X.stride(0) if M else w.K, _ptr(Y), Y.stride(0) if M else w.N,
                               _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_fp8_linear_grouped(w: Fp8Weights, X: torch.Tensor, off: torch.Tensor, Y: torch.Tensor,
                           workspace: torch.Tensor, stream=None):
    M = X.shape[0]
    _check(_lib.osc_fp8_linear_grouped(w.ptr, _ptr(X), _ptr(off), M, X.stride(0) if M else w.K, _ptr(Y),
                                       Y.stride(0) if M else w.N, _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream)))


# ------------------------------------------------------------- MXFP8 form of the fallback

def osc_mxfp8_weight_sizes(E: int, N: int, K: int) -> Mxfp8WeightSizes:
    out = Mxfp8WeightSizes()
    _check(_lib.osc_mxfp8_weight_sizes(E, N, K, C.byref(out)))
    return out


def osc_mxfp8_prepare_weights(W: torch.Tensor, stream=None) -> Mxfp8Weights:
    N, K = W.shape
    sz = osc_mxfp8_weight_sizes(1, N, K)
    bufs = {"w8": _alloc(sz.w8_bytes, W.device), "sfw": _alloc(sz.sfw_bytes, W.device)}
    h = _vp()
    _check(_lib.osc_mxfp8_prepare_weights(_ptr(W), N, K, W.stride(0), _ptr(bufs["w8"]), _ptr(bufs["sfw"]),
                                          _stream(stream), C.byref(h)))
    w = Mxfp8Weights(h.value, bufs)
    w.E, w.N, w.K, w.sizes = 1, N, K, sz
    return w


def osc_mxfp8_prepare_weights_grouped(W: torch.Tensor, stream=None) -> Mxfp8Weights:
    E, N, K = W.shape
    assert W.is_contiguous()
    sz = osc_mxfp8_weight_sizes(E, N, K)
    bufs = {"w8": _alloc(sz.w8_bytes, W.device), "sfw": _alloc(sz.sfw_bytes, W.device)}
    h = _vp()
    _check(_lib.osc_mxfp8_prepare_weights_grouped(_ptr(W), E, N, K, _ptr(bufs["w8"]), _ptr(bufs["sfw"]),
                                                  _stream(stream), C.byref(h)))
    w = Mxfp8Weights(h.value, bufs)
    w.E, w.N, w.K, w.sizes = E, N, K, sz
    return w


def osc_mxfp8_linear_grouped(w: Mxfp8Weights, X: torch.Tensor, off: torch.Tensor, Y: torch.Tensor,
                             workspace: torch.Tensor, stream=None):
    M = X.shape[0]
    _check(_lib.osc_mxfp8_linear_grouped(w.ptr, _ptr(X), _ptr(off), M, X.stride(0) if M else w.K, _ptr(Y),
                                         Y.stride(0) if M else w.N, _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_mxfp8_weights_destroy(w: Mxfp8Weights):
    w.close()


def osc_mxfp8_act_sizes(w: Mxfp8Weights, M: int) -> Mxfp8ActSizes:
    out = Mxfp8ActSizes()
    _check(_lib.osc_mxfp8_act_sizes(w.ptr, M, C.byref(out)))
    return out


def osc_mxfp8_quantize(X: torch.Tensor, x8, sfa, stream=None):
    M, K = X.shape
    _check(_lib.osc_mxfp8_quantize(_ptr(X), M, K, X.stride(0) if M else K, _ptr(x8), _ptr(sfa), _stream(stream)))


def osc_mxfp8_gemm(w: Mxfp8Weights, x8, sfa, M: int, Y: torch.Tensor, stream=None):
    _check(_lib.osc_mxfp8_gemm(w.ptr, _ptr(x8), _ptr(sfa), M, _ptr(Y), Y.stride(0) if M else w.N, _stream(stream)))


def osc_mxfp8_linear(w: Mxfp8Weights, X: torch.Tensor, Y: torch.Tensor, workspace: torch.Tensor, stream=None):
    M = X.shape[0]
    _check(_lib.osc_mxfp8_linear(w.ptr, _ptr(X), M, X.stride(0) if M else w.K, _ptr(Y), Y.stride(0) if M else w.N,
                                 _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


# ------------------------------------------- dynamic-protection control group (a baseline)

def osc_dyn_weight_sizes(N: int, K: int) -> WeightSizes:
    out = WeightSizes()
    _check(_lib.osc_dyn_weight_sizes(N, K, C.byref(out)))
    return out


def osc_dyn_prepare_weights(W: torch.Tensor, stream=None) -> OscWeights:
    N, K = W.shape
    sz = osc_dyn_weight_sizes(N, K)
    bufs = {k: _alloc(getattr(sz, k + "_bytes"), W.device) for k in ("wq", "sfw", "wo", "meta")}
    h = _vp()
    _check(_lib.osc_dyn_prepare_weights(_ptr(W), N, K, W.stride(0), _ptr(bufs["wq"]), _ptr(bufs["sfw"]),
                                        _ptr(bufs["wo"]), _ptr(bufs["meta"]), _stream(stream), C.byref(h)))
    w = OscWeights(h.value, bufs)
    w.E, w.N, w.K, w.K_o, w.K_o_pad, w.sizes = 1, N, K, K, K, sz
    return w


def osc_dyn_act_sizes(w: OscWeights, M: int) -> DynActSizes:
    out = DynActSizes()
    _check(_lib.osc_dyn_act_sizes(w.ptr, M, C.byref(out)))
    return out


def osc_dyn_quantize_extract(w: OscWeights, X: torch.Tensor, xq, sfa, xo, idx, val, stream=None):
    M = X.shape[0]
    _check(_lib.osc_dyn_quantize_extract(w.ptr, _ptr(X), M, X.stride(0) if M else w.K, _ptr(xq), _ptr(sfa), _ptr(xo),
                                         _ptr(idx), _ptr(val), _stream(stream)))


def osc_dyn_linear(w: OscWeights, X: torch.Tensor, Y: torch.Tensor, workspace: torch.Tensor, stream=None):
    M = X.shape[0]
    _check(_lib.osc_dyn_linear(w.ptr, _ptr(X), M, X.stride(0) if M else w.K, _ptr(Y), Y.stride(0) if M else w.N,
                               _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


# --------------------------------------------------------------- NVFP4 / G = 16 variant

def _lut16(lut, K):
    lut = np.ascontiguousarray(lut, dtype=np.int8)
    return lut.reshape(K // 16, -1)


def osc_nvfp4_weight_sizes(N: int, K: int, lut16) -> WeightSizes:
    lut16 = _lut16(lut16, K)
    out = WeightSizes()
    _check(_lib.osc_nvfp4_weight_sizes(N, K, lut16.ctypes.data, lut16.shape[1], C.byref(out)))
    return out


def osc_nvfp4_prepare_weights(W: torch.Tensor, lut16, ew: int, stream=None) -> OscWeights:
    N, K = W.shape
    lut16 = _lut16(lut16, K)
    sz = osc_nvfp4_weight_sizes(N, K, lut16)
    bufs = {k: _alloc(getattr(sz, k + "_bytes"), W.device) for k in ("wq", "sfw", "wo", "meta")}
    h = _vp()
    _check(_lib.osc_nvfp4_prepare_weights(_ptr(W), N, K, W.stride(0), lut16.ctypes.data, lut16.shape[1], int(ew),
                                          _ptr(bufs["wq"]), _ptr(bufs["sfw"]), _ptr(bufs["wo"]) if sz.wo_bytes else None,
                                          _ptr(bufs["meta"]), _stream(stream), C.byref(h)))
    w = OscWeights(h.value, bufs)
    w.E, w.N, w.K, w.K_o, w.K_o_pad, w.sizes, w.ew = 1, N, K, sz.K_o, sz.K_o_pad, sz, int(ew)
    return w


def osc_nvfp4_prepare_weights_grouped(W: torch.Tensor, lut16, ew: int, stream=None) -> OscWeights:
    """W: cuda bf16 [E, N, K] contiguous; one table and one tensor exponent for all experts."""
    E, N, K = W.shape
    assert W.is_contiguous()
    lut16 = _lut16(lut16, K)
    sz = WeightSizes()
    _check(_lib.osc_nvfp4_weight_sizes_grouped(E, N, K, lut16.ctypes.data, lut16.shape[1], C.byref(sz)))
    bufs = {k: _alloc(getattr(sz, k + "_bytes"), W.device) for k in ("wq", "sfw", "wo", "meta")}
    h = _vp()
    _check(_lib.osc_nvfp4_prepare_weights_grouped(_ptr(W), E, N, K, lut16.ctypes.data, lut16.shape[1], int(ew),
                                                  _ptr(bufs["wq"]), _ptr(bufs["sfw"]),
                                                  _ptr(bufs["wo"]) if sz.wo_bytes else None, _ptr(bufs["meta"]),
                                                  _stream(stream), C.byref(h)))
    w = OscWeights(h.value, bufs)
    w.E, w.N, w.K, w.K_o, w.K_o_pad, w.sizes, w.ew = E, N, K, sz.K_o, sz.K_o_pad, sz, int(ew)
    return w


def osc_nvfp4_linear_grouped(w: OscWeights, X: torch.Tensor, off: torch.Tensor, ex: int, Y: torch.Tensor,
                             workspace: torch.Tensor, stream=None):
    M = X.shape[0]
    _check(_lib.osc_nvfp4_linear_grouped(w.ptr, _ptr(X), _ptr(off), M, X.stride(0) if M else w.K, int(ex), _ptr(Y),
                                         Y.stride(0) if M else w.N, _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_nvfp4_act_sizes(w: OscWeights, M: int) -> ActSizes:
    out = ActSizes()
    _check(_lib.osc_nvfp4_act_sizes(w.ptr, M, C.byref(out)))
    return out


def osc_nvfp4_quantize_extract(w: OscWeights, X: torch.Tensor, ex: int, xq, sfa, xo, stream=None):
    M = X.shape[0]
    _check(_lib.osc_nvfp4_quantize_extract(w.ptr, _ptr(X), M, X.stride(0) if M else w.K, int(ex), _ptr(xq), _ptr(sfa),
                                           _ptr(xo) if w.K_o_pad else None, _stream(stream)))


def osc_nvfp4_gemm(w: OscWeights, xq, sfa, xo, M: int, ex: int, Y: torch.Tensor, stream=None):
    _check(_lib.osc_nvfp4_gemm(w.ptr, _ptr(xq), _ptr(sfa), _ptr(xo) if w.K_o_pad else None, M, int(ex), _ptr(Y),
                               Y.stride(0) if M else w.N, _stream(stream)))


def osc_nvfp4_linear(w: OscWeights, X: torch.Tensor, ex: int, Y: torch.Tensor, workspace: torch.Tensor, stream=None):
    M = X.shape[0]
    _check(_lib.osc_nvfp4_linear(w.ptr, _ptr(X), M, X.stride(0) if M else w.K, int(ex), _ptr(Y),
                                 Y.stride(0) if M else w.N, _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_nvfp4_rmsnorm_quantize_extract(w: OscWeights, H: torch.Tensor, gamma: torch.Tensor, eps: float, ex: int, xq, sfa, xo,
                                       stream=None):
    M = H.shape[0]
    _check(_lib.osc_nvfp4_rmsnorm_quantize_extract(w.ptr, _ptr(H), M, H.stride(0) if M else w.K, _ptr(gamma), float(eps),
                                                   int(ex), _ptr(xq), _ptr(sfa), _ptr(xo) if w.K_o_pad else None,
                                                   _stream(stream)))


def osc_nvfp4_rmsnorm_linear(w: OscWeights, H: torch.Tensor, gamma: torch.Tensor, eps: float, ex: int, Y: torch.Tensor,
                             workspace: torch.Tensor, stream=None):
    M = H.shape[0]
    _check(_lib.osc_nvfp4_rmsnorm_linear(w.ptr, _ptr(H), M, H.stride(0) if M else w.K, _ptr(gamma), float(eps), int(ex),
                                         _ptr(Y), Y.stride(0) if M else w.N, _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_nvfp4_gather_workspace_bytes(w: OscWeights, T: int, M_total: int) -> int:
    out = _sz()
    _check(_lib.osc_nvfp4_gather_workspace_bytes(w.ptr, T, M_total, C.byref(out)))
    return int(out.value)


def osc_nvfp4_linear_grouped_gather(w: OscWeights, X: torch.Tensor, row_token: torch.Tensor, off: torch.Tensor, ex: int,
                                    Y: torch.Tensor, workspace: torch.Tensor, stream=None):
    T, M = X.shape[0], row_token.shape[0]
    _check(_lib.osc_nvfp4_linear_grouped_gather(w.ptr, _ptr(X), T, X.stride(0) if T else w.K, _ptr(row_token), _ptr(off), M,
                                                int(ex), _ptr(Y), Y.stride(0) if M else w.N, _ptr(workspace),
                                                workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_nvfp4_rmsnorm_linear_grouped_gather(w: OscWeights, H: torch.Tensor, gamma: torch.Tensor, eps: float,
                                            row_token: torch.Tensor, off: torch.Tensor, ex: int, Y: torch.Tensor,
                                            workspace: torch.Tensor, stream=None):
    T, M = H.shape[0], row_token.shape[0]
    _check(_lib.osc_nvfp4_rmsnorm_linear_grouped_gather(w.ptr, _ptr(H), T, H.stride(0) if T else w.K, _ptr(gamma), float(eps),
                                                        _ptr(row_token), _ptr(off), M, int(ex), _ptr(Y),
                                                        Y.stride(0) if M else w.N, _ptr(workspace),
                                                        workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_prepare_weights_gate_up(W: torch.Tensor, lut, stream=None) -> OscWeights:
    """W: cuda bf16 [2I, K], gate rows above up rows.  A dense OSC handle that also serves osc_linear_swiglu."""
    N, K = W.shape
    I = N // 2
    lut = _lut(lut)
    sz = WeightSizes()
    _check(_lib.osc_gate_up_weight_sizes(I, K, lut.ctypes.data, lut.shape[1], C.byref(sz)))
    bufs = {k: _alloc(getattr(sz, k + "_bytes"), W.device) for k in ("wq", "sfw", "wo", "meta")}
    h = _vp()
    _check(_lib.osc_prepare_weights_gate_up(_ptr(W), I, K, W.stride(0), lut.ctypes.data, lut.shape[1], _ptr(bufs["wq"]),
                                            _ptr(bufs["sfw"]), _ptr(bufs["wo"]) if sz.wo_bytes else None, _ptr(bufs["meta"]),
                                            _stream(stream), C.byref(h)))
    w = OscWeights(h.value, bufs)
    w.E, w.N, w.K, w.K_o, w.K_o_pad, w.sizes = 1, N, K, sz.K_o, sz.K_o_pad, sz
    return w


def osc_linear_swiglu_workspace_bytes(w: OscWeights, M: int) -> int:
    out = _sz()
    _check(_lib.osc_linear_swiglu_workspace_bytes(w.ptr, M, C.byref(out)))
    return int(out.value)


def osc_linear_swiglu(w: OscWeights, X: torch.Tensor, H: torch.Tensor, workspace: torch.Tensor, stream=None):
    """H [M, I] = silu(gate) * up of the gate|up projection of X, the activation applied in the GEMM epilogue."""
    M = X.shape[0]
    _check(_lib.osc_linear_swiglu(w.ptr, _ptr(X), M, X.stride(0) if M else w.K, _ptr(H), H.stride(0) if M else w.N // 2,
                                  _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_rmsnorm_linear_swiglu(w: OscWeights, Hin: torch.Tensor, gamma: torch.Tensor, eps: float, H: torch.Tensor,
                              workspace: torch.Tensor, stream=None):
    M = Hin.shape[0]
    _check(_lib.osc_rmsnorm_linear_swiglu(w.ptr, _ptr(Hin), M, Hin.stride(0) if M else w.K, _ptr(gamma), float(eps), _ptr(H),
                                          H.stride(0) if M else w.N // 2, _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_prepare_weights_gate_up_grouped(W: torch.Tensor, lut, stream=None) -> OscWeights:
    """W: cuda bf16 [E, 2I, K] contiguous, every expert's gate rows above its up rows."""
    E, N, K = W.shape
    assert W.is_contiguous()
    lut = _lut(lut)
    sz = WeightSizes()
    _check(_lib.osc_gate_up_weight_sizes_grouped(E, N // 2, K, lut.ctypes.data, lut.shape[1], C.byref(sz)))
    bufs = {k: _alloc(getattr(sz, k + "_bytes"), W.device) for k in ("wq", "sfw", "wo", "meta")}
    h = _vp()
    _check(_lib.osc_prepare_weights_gate_up_grouped(_ptr(W), E, N // 2, K, lut.ctypes.data, lut.shape[1], _ptr(bufs["wq"]),
                                                    _ptr(bufs["sfw"]), _ptr(bufs["wo"]) if sz.wo_bytes else None,
                                                    _ptr(bufs["meta"]), _stream(stream), C.byref(h)))
    w = OscWeights(h.value, bufs)
    w.E, w.N, w.K, w.K_o, w.K_o_pad, w.sizes = E, N, K, sz.K_o, sz.K_o_pad, sz
    return w


def osc_linear_swiglu_grouped(w: OscWeights, X: torch.Tensor, off: torch.Tensor, H: torch.Tensor, workspace: torch.Tensor,
                              stream=None):
    M = X.shape[0]
    _check(_lib.osc_linear_swiglu_grouped(w.ptr, _ptr(X), _ptr(off), M, X.stride(0) if M else w.K, _ptr(H),
                                          H.stride(0) if M else w.N // 2, _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_swiglu_gather_workspace_bytes(w: OscWeights, T: int, M_total: int) -> int:
    out = _sz()
    _check(_lib.osc_swiglu_gather_workspace_bytes(w.ptr, T, M_total, C.byref(out)))
    return int(out.value)


def osc_linear_swiglu_grouped_gather(w: OscWeights, X: torch.Tensor, row_token: torch.Tensor, off: torch.Tensor, H: torch.Tensor,
                                     workspace: torch.Tensor, stream=None):
    T, M = X.shape[0], row_token.shape[0]
    _check(_lib.osc_linear_swiglu_grouped_gather(w.ptr, _ptr(X), T, X.stride(0) if T else w.K, _ptr(row_token), _ptr(off), M,
                                                 _ptr(H), H.stride(0) if M else w.N // 2, _ptr(workspace),
                                                 workspace.numel() * workspace.element_size(), _stream(stream)))


def osc_rmsnorm_linear_swiglu_grouped_gather(w: OscWeights, Hin: torch.Tensor, gamma: torch.Tensor, eps: float,
                                             row_token: torch.Tensor, off: torch.Tensor, H: torch.Tensor, workspace: torch.Tensor,
                                             stream=None):
    T, M = Hin.shape[0], row_token.shape[0]
    _check(_lib.osc_rmsnorm_linear_swiglu_grouped_gather(w.ptr, _ptr(Hin), T, Hin.stride(0) if T else w.K, _ptr(gamma),
                                                         float(eps), _ptr(row_token), _ptr(off), M, _ptr(H),
                                                         H.stride(0) if M else w.N // 2, _ptr(workspace),
                                                         workspace.numel() * workspace.element_size(), _stream(stream)))


# ------------------------------- between the QKV projection and o_proj: a paged key/value cache

# Lengths, tables and slots are read on the device, where a tensor of another type or on another device would go unnoticed, so the calls
# below look at every tensor.  They run once per step or layer in front of kernels of a few microseconds: the look is one pass with three
# attribute reads a tensor, and only a refusal works out what was wrong.  (t.stride()[0]: half the time of t.stride(0).)
def _device_of(t):
    """Device of a call: that of its first tensor, which has to be the current one; -1 otherwise."""
    d = t.get_device()
    return d if d >= 0 and d == (_raw_device() if _raw_device is not None else torch.cuda.current_device()) else -1


def _refuse(dtype, ndim, dev, **tensors):
    for name, t in tensors.items():
        if t is None:
            continue
        if t.dtype != dtype or (ndim and t.dim() != ndim):
            raise ValueError(f"{name}: {ndim if ndim else 'any'}-d {dtype} expected, got {t.dim()}-d {t.dtype}")
        if not t.is_cuda:
            raise ValueError(f"{name}: cuda tensor expected")
        if dev < 0 or t.get_device() != dev:
            raise ValueError(f"{name}: lies on {t.device}, not on the current device")
        if t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}: the last dimension must be contiguous")


def _bad(dtype, dev, *tensors):
    """Whether a call must not take one of these (one-dimensional or wholly contiguous) tensors."""
    for t in tensors:
        if t is not None and (t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous()):
            return True
    return dev < 0


def _bad_rows(dtype, dev, *tensors):
    """The same for matrices whose rows may be further apart than they are long."""
    for t in tensors:
        if t is not None and (t.dtype is not dtype or t.get_device() != dev or t.dim() != 2 or (t.stride()[1] != 1 and t.shape[1] > 1)):
            return True
    return dev < 0


def _addr(t):
    return t.data_ptr() if t is not None else None


class KvCache:
    """Keys and values of one layer: cuda bf16 [n_pages, page_size, n_heads, head_dim] views, any strides that leave the
    channels contiguous (a permuted [n_pages, n_heads, page_size, head_dim] buffer too), the same for k and v."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        _refuse(torch.bfloat16, 4, k.get_device(), k=k, v=v)
        if k.shape != v.shape or any(a != b for n, a, b in zip(k.shape, k.stride(), v.stride()) if n > 1):
            raise ValueError("k and v must have the same shape and strides")
        self.k, self.v, self.device = k, v, k.get_device()
        n_pages, page_size, n_heads, head_dim = k.shape
        st = [s if n > 1 else 8 * ((head_dim + 7) // 8) for n, s in zip(k.shape[:3], k.stride()[:3])]
        self.n_pages, self.page_size, self.n_heads, self.head_dim = n_pages, page_size, n_heads, head_dim
        self.c = KvCacheStruct(_ptr(k), _ptr(v), n_pages, page_size, n_heads, head_dim, *st)


class Rope:
    """Rotation by position: inv_freq cuda float32 [rot_dim / 2]; axis cuda uint8 [rot_dim / 2] (which of the position
    axes turns a pair) or None."""

    def __init__(self, inv_freq: torch.Tensor, axis: torch.Tensor = None, interleaved: bool = False, scale: float = 1.0):
        _refuse(torch.float32, 1, inv_freq.get_device(), inv_freq=inv_freq)
        _refuse(torch.uint8, 1, inv_freq.get_device(), axis=axis)
        if axis is not None and axis.shape != inv_freq.shape:
            raise ValueError("axis and inv_freq must have the same length")
        self.inv_freq, self.axis, self.interleaved, self.scale, self.device = inv_freq, axis, interleaved, scale, inv_freq.get_device()
        self.c = {n: RopeStruct(_ptr(inv_freq), _ptr(axis), 2 * inv_freq.shape[0], n, int(interleaved), scale) for n in (1, 2, 3)}


def osc_kv_slots(cached, fresh, base, page_size: int, free_pages, table, row_off, kv_len, slots, positions, taken, stream=None):
    """Pages, slots and positions of a step's new tokens from the requests' lengths (all int32; table [R, cols] is
    updated in place, row_off [R + 1], kv_len [R], slots [T], positions [T] and taken [1] are written)."""
    dev, i32 = _device_of(cached), torch.int32
    if _bad(i32, dev, cached, fresh, base, free_pages, row_off, kv_len, slots, positions, taken) or _bad_rows(i32, dev, table):
        _refuse(i32, 1, dev, cached=cached, fresh=fresh, base=base, free_pages=free_pages, row_off=row_off, kv_len=kv_len, slots=slots,
                positions=positions, taken=taken)
        _refuse(i32, 2, dev, table=table)
    R, T = cached.numel(), slots.numel()
    rows, cols = table.shape
    if (fresh.numel() != R or rows != R or kv_len.numel() < R or row_off.numel() < R + 1 or positions.numel() < T or taken.numel() < 1 or
            (base is not None and base.numel() != R)):
        raise ValueError("osc_kv_slots: lengths do not belong together")
    _check(_lib.osc_kv_slots(cached.data_ptr(), fresh.data_ptr(), _addr(base), R, page_size, free_pages.data_ptr(), free_pages.numel(),
                             table.data_ptr(), cols, table.stride()[0], T, row_off.data_ptr(), kv_len.data_ptr(), slots.data_ptr(),
                             positions.data_ptr(), taken.data_ptr(), _stream(stream)))


def osc_qk_norm_rope(QKV: torch.Tensor, n_q: int, cache: KvCache, Q: torch.Tensor, positions: torch.Tensor, rope: Rope, gamma_q=None,
                     gamma_k=None, eps: float = 1e-6, slots=None, stream=None):
    """Norm and rotation of the query and key heads of QKV [T, (n_q + 2 n_kv) head_dim]; queries to Q [T, n_q head_dim],
    keys and values to their slots of the cache.  positions: int32 [T] or [axes, T]."""
    dev, i32, bf16 = _device_of(QKV), torch.int32, torch.bfloat16
    two = positions.dim() == 2
    if (_bad_rows(bf16, dev, QKV, Q) or _bad(bf16, dev, gamma_q, gamma_k) or _bad(i32, dev, slots) or
            (_bad_rows if two else _bad)(i32, dev, positions) or cache.device != dev or rope.device != dev):
        _refuse(bf16, 2, dev, QKV=QKV, Q=Q)
        _refuse(bf16, 1, dev, gamma_q=gamma_q, gamma_k=gamma_k)
        _refuse(i32, 1, dev, slots=slots)
        _refuse(i32, 2 if two else 1, dev, positions=positions)
        raise ValueError(f"osc_qk_norm_rope: cache on cuda:{cache.device}, rope on cuda:{rope.device}, QKV on cuda:{dev}; vectors must be contiguous")
    T, width = QKV.shape
    qT, qw = Q.shape
    axes = positions.shape[0] if two else 1
    if not 1 <= axes <= 3:
        raise ValueError("positions: [T] or [axes, T] with at most three axes")
    if (positions.shape[-1] < T or qT != T or (slots is not None and slots.numel() < T) or
            width != (n_q + 2 * cache.n_heads) * cache.head_dim or qw < n_q * cache.head_dim or
            (gamma_q is not None and gamma_q.numel() != cache.head_dim) or (gamma_k is not None and gamma_k.numel() != cache.head_dim)):
        raise ValueError("osc_qk_norm_rope: shapes do not belong together")
    _check(_lib.osc_qk_norm_rope(QKV.data_ptr(), T, QKV.stride()[0] if T > 1 else width, n_q, cache.c, _addr(gamma_q), _addr(gamma_k), eps,
                                 rope.c[axes], positions.data_ptr(), positions.stride()[0] if axes > 1 else T, _addr(slots), Q.data_ptr(),
                                 Q.stride()[0] if T > 1 else qw, _stream(stream)))


def osc_paged_attention_workspace_bytes(T: int, n_q: int, head_dim: int, R: int, P: int = 0) -> int:
    out = _sz()
    _check(_lib.osc_paged_attention_workspace_bytes(T, n_q, head_dim, R, P, C.byref(out)))
    return int(out.value)


def osc_paged_attention(Q: torch.Tensor, cache: KvCache, row_off, kv_len, table, O: torch.Tensor, workspace: torch.Tensor, scale: float,
                        lse=None, group_off=None, prefix_len=None, prefix_table=None, max_new: int = 0, stream=None):
    """Attention of the new tokens Q [T, n_q head_dim] over the cache; O [T, n_q head_dim], lse float32 [T, n_q] or None.
    With group_off [P + 1], prefix_len [P] and prefix_table [P, cols], groups of requests share prefixes."""
    dev, i32, bf16 = _device_of(Q), torch.int32, torch.bfloat16
    if (_bad_rows(bf16, dev, Q, O) or _bad(i32, dev, row_off, kv_len, prefix_len, group_off) or _bad_rows(i32, dev, table, prefix_table) or
            _bad(torch.float32, dev, lse) or _bad(torch.uint8, dev, workspace) or cache.device != dev):
        _refuse(bf16, 2, dev, Q=Q, O=O)
        _refuse(i32, 1, dev, row_off=row_off, kv_len=kv_len, prefix_len=prefix_len, group_off=group_off)
        _refuse(i32, 2, dev, table=table, prefix_table=prefix_table)
        _refuse(torch.float32, 2, dev, lse=lse)
        _refuse(torch.uint8, 1, dev, workspace=workspace)
        raise ValueError(f"osc_paged_attention: vectors and lse must be contiguous, the cache (cuda:{cache.device}) on the device of Q, cuda:{dev}")
    T, width = Q.shape
    R, (rows, cols), n_q = kv_len.numel(), table.shape, width // cache.head_dim
    P = prefix_len.numel() if prefix_len is not None else 0
    if (width % cache.head_dim or O.shape != Q.shape or row_off.numel() < R + 1 or rows < R or
            (P and (group_off is None or prefix_table is None or group_off.numel() < P + 1 or prefix_table.shape[0] < P)) or
            (lse is not None and lse.numel() != T * n_q)):
        raise ValueError("osc_paged_attention: shapes do not belong together")
    ldq, ldo = (Q.stride()[0], O.stride()[0]) if T > 1 else (width, width)
    if P:
        _check(_lib.osc_paged_attention(Q.data_ptr(), T, ldq, n_q, cache.c, R, row_off.data_ptr(), kv_len.data_ptr(), table.data_ptr(), cols,
                                        table.stride()[0], P, group_off.data_ptr(), prefix_len.data_ptr(), prefix_table.data_ptr(),
                                        prefix_table.shape[1], prefix_table.stride()[0], max_new, scale, O.data_ptr(), ldo, _addr(lse),
                                        workspace.data_ptr(), workspace.numel(), _stream(stream)))
    else:
        _check(_lib.osc_paged_attention(Q.data_ptr(), T, ldq, n_q, cache.c, R, row_off.data_ptr(), kv_len.data_ptr(), table.data_ptr(), cols,
                                        table.stride()[0], 0, None, None, None, 0, 0, max_new, scale, O.data_ptr(), ldo, _addr(lse),
                                        workspace.data_ptr(), workspace.numel(), _stream(stream)))


class KvLayers:
    """The caches of a model's layers (KvCache, all of one shape and strides), for calls that move tokens in all of them."""

    def __init__(self, caches):
        self.caches = list(caches)
        if not self.caches:
            raise ValueError("KvLayers: no cache")
        self.first = self.caches[0]
        self.device = self.first.device
        if any(c.device != self.device for c in self.caches):
            raise ValueError("KvLayers: caches on several devices")
        self.c = (KvCacheStruct * len(self.caches))(*[c.c for c in self.caches])

    def __len__(self):
        return len(self.caches)


def osc_tree_mask(parents, row_off, base, mask, positions=None, stream=None):
    """Ancestors (mask [T, words], bits) and positions [T] of drafted tokens from their parents [T]; row_off [R + 1], base [R] or None.  All int32."""
    dev, i32 = _device_of(parents), torch.int32
    if _bad(i32, dev, parents, row_off, base, positions) or _bad_rows(i32, dev, mask):
        _refuse(i32, 1, dev, parents=parents, row_off=row_off, base=base, positions=positions)
        _refuse(i32, 2, dev, mask=mask)
        raise ValueError("osc_tree_mask: vectors must be contiguous")
    T, R = parents.numel(), row_off.numel() - 1
    rows, words = mask.shape
    if R < 0 or rows != T or (base is not None and base.numel() < R) or (positions is not None and positions.numel() < T):
        raise ValueError("osc_tree_mask: lengths do not belong together")
    _check(_lib.osc_tree_mask(parents.data_ptr(), row_off.data_ptr(), _addr(base), R, T, mask.data_ptr(), words, mask.stride()[0] if T > 1 else words,
                              _addr(positions), _stream(stream)))


def osc_tree_attention(Q: torch.Tensor, cache: KvCache, row_off, kv_len, table, mask, O: torch.Tensor, workspace: torch.Tensor, scale: float,
                       lse=None, group_off=None, prefix_len=None, prefix_table=None, max_new: int = 0, stream=None):
    """osc_paged_attention with a mask among the new tokens: int32 [T, words], bit m of a token's row set where it sees its request's new token m."""
    dev, i32, bf16 = _device_of(Q), torch.int32, torch.bfloat16
    if (_bad_rows(bf16, dev, Q, O) or _bad(i32, dev, row_off, kv_len, prefix_len, group_off) or _bad_rows(i32, dev, table, prefix_table, mask) or
            _bad(torch.float32, dev, lse) or _bad(torch.uint8, dev, workspace) or cache.device != dev):
        _refuse(bf16, 2, dev, Q=Q, O=O)
        _refuse(i32, 1, dev, row_off=row_off, kv_len=kv_len, prefix_len=prefix_len, group_off=group_off)
        _refuse(i32, 2, dev, table=table, prefix_table=prefix_table, mask=mask)
        _refuse(torch.float32, 2, dev, lse=lse)
        _refuse(torch.uint8, 1, dev, workspace=workspace)
        raise ValueError(f"osc_tree_attention: vectors and lse must be contiguous, the cache (cuda:{cache.device}) on the device of Q, cuda:{dev}")
    T, width = Q.shape
    R, (rows, cols), n_q = kv_len.numel(), table.shape, width // cache.head_dim
    P = prefix_len.numel() if prefix_len is not None else 0
    if (width % cache.head_dim or O.shape != Q.shape or row_off.numel() < R + 1 or rows < R or mask.shape[0] != T or
            (P and (group_off is None or prefix_table is None or group_off.numel() < P + 1 or prefix_table.shape[0] < P)) or
            (lse is not None and lse.numel() != T * n_q)):
        raise ValueError("osc_tree_attention: shapes do not belong together")
    words = mask.shape[1]
    ldq, ldo, ldm = (Q.stride()[0], O.stride()[0], mask.stride()[0]) if T > 1 else (width, width, words)
    prefix = (P, group_off.data_ptr(), prefix_len.data_ptr(), prefix_table.data_ptr(), prefix_table.shape[1],
              prefix_table.stride()[0]) if P else (0, None, None, None, 0, 0)
    _check(_lib.osc_tree_attention(Q.data_ptr(), T, ldq, n_q, cache.c, R, row_off.data_ptr(), kv_len.data_ptr(), table.data_ptr(), cols,
                                   table.stride()[0], *prefix, mask.data_ptr(), words, ldm, max_new, scale, O.data_ptr(), ldo, _addr(lse),
                                   workspace.data_ptr(), workspace.numel(), _stream(stream)))


def osc_token_logprobs(logits: torch.Tensor, ids=None, logprob=None, scale: float = 1.0, lse=None, entropy=None, top_ids=None, top_logprobs=None,
                       stream=None):
    """Log probabilities (float32 [T, n_ids]) of the given tokens (int32 [T, n_ids]) under logits (bf16 or float32 [T, V]) times scale; lse and
    entropy float32 [T]; the best alternatives, top_ids int32 [T, k] and top_logprobs float32 [T, k].  What is None is left out."""
    dev, i32, f32 = _device_of(logits), torch.int32, torch.float32
    if logits.dtype not in (torch.bfloat16, f32):
        raise ValueError(f"osc_token_logprobs: logits are {logits.dtype}, must be bfloat16 or float32")
    if _bad_rows(logits.dtype, dev, logits) or _bad_rows(i32, dev, ids) or _bad(i32, dev, top_ids) or _bad(f32, dev, logprob, lse, entropy, top_logprobs):
        _refuse(logits.dtype, 2, dev, logits=logits)
        _refuse(i32, 2, dev, ids=ids, top_ids=top_ids)
        _refuse(f32, 2, dev, logprob=logprob, top_logprobs=top_logprobs)
        _refuse(f32, 1, dev, lse=lse, entropy=entropy)
        raise ValueError("osc_token_logprobs: what is written must be contiguous")
    T, V = logits.shape
    n_ids, k = ids.shape[1] if ids is not None else 0, top_ids.shape[1] if top_ids is not None else 0
    if ((ids is None) != (logprob is None) or (ids is not None and (ids.shape[0] != T or logprob.shape != ids.shape)) or
            (top_ids is None) != (top_logprobs is None) or (top_ids is not None and (top_ids.shape[0] != T or top_logprobs.shape != top_ids.shape)) or
            (lse is not None and lse.numel() != T) or (entropy is not None and entropy.numel() != T)):
        raise ValueError("osc_token_logprobs: shapes do not belong together")
    ld, ld_ids = (logits.stride()[0], ids.stride()[0] if ids is not None else 0) if T > 1 else (V, n_ids)
    _check(_lib.osc_token_logprobs(logits.data_ptr(), 1 if logits.dtype is f32 else 0, T, V, ld, scale, _addr(ids), n_ids, ld_ids, _addr(logprob),
                                   _addr(lse), _addr(entropy), k, _addr(top_ids), _addr(top_logprobs), _stream(stream)))


def osc_kv_compact(layers: KvLayers, row_off, kv_len, table, keep, n_keep, new_len, stream=None):
    """Accepted tokens moved together in all layers: keep [R, most] indices among the new tokens, n_keep [R] of them; new_len [R] is written.  All int32."""
    dev, i32 = _device_of(kv_len), torch.int32
    if _bad(i32, dev, row_off, kv_len, n_keep, new_len) or _bad_rows(i32, dev, table, keep) or layers.device != dev:
        _refuse(i32, 1, dev, row_off=row_off, kv_len=kv_len, n_keep=n_keep, new_len=new_len)
        _refuse(i32, 2, dev, table=table, keep=keep)
        raise ValueError(f"osc_kv_compact: vectors must be contiguous, the layers (cuda:{layers.device}) on the device of kv_len, cuda:{dev}")
    R = kv_len.numel()
    if row_off.numel() < R + 1 or n_keep.numel() != R or new_len.numel() < R or table.shape[0] < R or keep.shape[0] != R:
        raise ValueError("osc_kv_compact: lengths do not belong together")
    _check(_lib.osc_kv_compact(layers.c, len(layers.caches), R, row_off.data_ptr(), kv_len.data_ptr(), table.data_ptr(), table.shape[1], table.stride()[0],
                               keep.data_ptr(), keep.shape[1], keep.stride()[0], n_keep.data_ptr(), new_len.data_ptr(), _stream(stream)))


def osc_kv_trim(from_len, to_len, page_size: int, table, refs, freed, n_freed, n_pages: int = None, stream=None):
    """Pages given back by requests that shrink from from_len to to_len [R] tokens; table [R, cols] and refs [n_pages] (or None) are updated in place,
    freed [n_pages] and n_freed [1] are written.  All int32.  n_pages: the length of refs, or of freed without it, if it is not given.  (refs of pages that
    osc_kv_slots took are the caller's to raise.)"""
    dev, i32 = _device_of(from_len), torch.int32
    if _bad(i32, dev, from_len, to_len, refs, freed, n_freed) or _bad_rows(i32, dev, table):
        _refuse(i32, 1, dev, from_len=from_len, to_len=to_len, refs=refs, freed=freed, n_freed=n_freed)
        _refuse(i32, 2, dev, table=table)
        raise ValueError("osc_kv_trim: vectors must be contiguous")
    R, (rows, cols) = from_len.numel(), table.shape
    if n_pages is None:
        n_pages = refs.numel() if refs is not None else freed.numel()
    if to_len.numel() != R or rows < R or (refs is not None and refs.numel() < n_pages) or freed.numel() < n_pages or n_freed.numel() < 1:
        raise ValueError("osc_kv_trim: lengths do not belong together")
    _check(_lib.osc_kv_trim(from_len.data_ptr(), to_len.data_ptr(), R, page_size, table.data_ptr(), cols, table.stride()[0], _addr(refs), n_pages,
                            freed.data_ptr(), n_freed.data_ptr(), _stream(stream)))


def osc_kv_fork(src, dst, len_, page_size: int, free_pages, table, refs, copy_from, copy_to, copy_used, taken, n_pages: int = None, stream=None):
    """Rows dst [n] of table [R, cols] become forks of rows src [n]; len_ [R], table and refs [n_pages] (or None, then n_pages is given) are updated in
    place, copy_from, copy_to, copy_used [n] (what osc_kv_copy_pages takes) and taken [1] are written.  All int32."""
    dev, i32 = _device_of(src), torch.int32
    if _bad(i32, dev, src, dst, len_, free_pages, refs, copy_from, copy_to, copy_used, taken) or _bad_rows(i32, dev, table):
        _refuse(i32, 1, dev, src=src, dst=dst, len_=len_, free_pages=free_pages, refs=refs, copy_from=copy_from, copy_to=copy_to, copy_used=copy_used,
                taken=taken)
        _refuse(i32, 2, dev, table=table)
        raise ValueError("osc_kv_fork: vectors must be contiguous")
    n, (R, cols) = src.numel(), table.shape
    if n_pages is None:
        if refs is None:
            raise ValueError("osc_kv_fork: n_pages is needed where there is no refs")
        n_pages = refs.numel()
    if (dst.numel() != n or len_.numel() < R or copy_from.numel() < n or copy_to.numel() < n or copy_used.numel() < n or taken.numel() < 1 or
            (refs is not None and refs.numel() < n_pages)):
        raise ValueError("osc_kv_fork: lengths do not belong together")
    _check(_lib.osc_kv_fork(src.data_ptr(), dst.data_ptr(), n, len_.data_ptr(), R, page_size, free_pages.data_ptr(), free_pages.numel(), table.data_ptr(), cols,
                            table.stride()[0], _addr(refs), n_pages, copy_from.data_ptr(), copy_to.data_ptr(), copy_used.data_ptr(), taken.data_ptr(),
                            _stream(stream)))


def osc_kv_copy_pages(layers: KvLayers, from_pages, to_pages, used=None, stream=None):
    """The first used[i] places (all without it) of page from_pages[i] to page to_pages[i], in all layers.  All int32 [n]."""
    dev, i32 = _device_of(from_pages), torch.int32
    if _bad(i32, dev, from_pages, to_pages, used) or layers.device != dev:
        _refuse(i32, 1, dev, from_pages=from_pages, to_pages=to_pages, used=used)
        raise ValueError(f"osc_kv_copy_pages: vectors must be contiguous, the layers (cuda:{layers.device}) on the device of from_pages, cuda:{dev}")
    n = from_pages.numel()
    if to_pages.numel() != n or (used is not None and used.numel() != n):
        raise ValueError("osc_kv_copy_pages: lengths do not belong together")
    _check(_lib.osc_kv_copy_pages(layers.c, len(layers.caches), from_pages.data_ptr(), to_pages.data_ptr(), _addr(used), n, _stream(stream)))

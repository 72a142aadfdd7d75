"""Thin Python binding over libapb.so (argument marshalling only).

Every step of the APB layer forward pass runs in the HIP kernels of the library; PyTorch is
used for device memory and streams, nothing else.  There is no CPU fallback: if the library
is missing or cannot be loaded, importing this module's functions raises.

Function names and argument order follow include/apb.h.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libapb.so")

EXPORTS = (
    "apb_compress", "apb_layer_info", "apb_layer_export", "apb_layer_free", "apb_acts_bytes",
    "apb_quantize_acts", "apb_forward", "apb_forward_kernel_name", "apb_quantize_forward", "apb_quantize_forward_static", "apb_quantize_forward_is_one_kernel", "apb_forward_requant", "apb_forward_conv3x3", "apb_forward_conv3x3_requant",
    "apb_layer_export_steps", "apb_forward_int", "apb_forward_int_popcount", "apb_forward_popcount",
    "apb_w2_pack", "apb_w2_export", "apb_w2_free", "apb_gemm_2_2_int", "apb_gemm_2_2",
    "apb_train_workspace_bytes", "apb_train_forward", "apb_train_backward",
    "apb_probe_out_bytes", "apb_probe_rate",
    "apb_mx4_bytes", "apb_mx4_quantize", "apb_mx4_dequantize", "apb_mx4_gemm", "apb_mx4_linear", "apb_mx4_linear_scratch_bytes",
    "apb_mx4_backward_input", "apb_mx4_backward_weight", "apb_mx4_backward_input_workspace_bytes",
    "apb_mx4_backward_weight_workspace_bytes",
    "apb_moe_workspace_bytes", "apb_moe_route", "apb_moe_route_backward", "apb_moe_combine", "apb_moe_combine_backward",
    "apb_mx8_bytes", "apb_mx8_quantize", "apb_mx8_dequantize", "apb_mx4_gated_gemm", "apb_mx4_gated_linear",
    "apb_mx4_gated_linear_scratch_bytes", "apb_gated_forward", "apb_gated_backward",
    "apb_adapter_parts", "apb_adapter_down", "apb_adapter_up", "apb_adapter_gradient", "apb_adapter_gradient_workspace_bytes",
    "apb_strerror", "apb_last_hip_error",
)

APB_OK = 0
APB_ERR_NULL, APB_ERR_SHAPE, APB_ERR_BITS, APB_ERR_VALUE, APB_ERR_NOMEM, APB_ERR_HIP = -1, -2, -3, -4, -5, -6
APB_ERR_SCRATCH, APB_ERR_TYPE, APB_ERR_ALIGN = -7, -8, -9
APB_STATIC_SCRATCH_BYTES = 32 << 20

_lib: Optional[ctypes.CDLL] = None
_several_devices = False                                              # (known once the library is loaded)


class ApbError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {strerror(code)} (status {code})")
        self.code = code


def load() -> ctypes.CDLL:
    """Load libapb.so; raises if it has not been built (python paper_2306_08960_amd/build.py)."""
    global _lib, _several_devices
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python {os.path.join(_HERE, 'build.py')}` "
                           "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    _several_devices = torch.cuda.device_count() > 1
    vp, ci, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    lib.apb_compress.argtypes = [vp, ci, ci, cf, cf, vp, ctypes.POINTER(vp)]
    lib.apb_compress.restype = ci
    lib.apb_layer_info.argtypes = [vp, ctypes.POINTER(ci), ctypes.POINTER(ci), ctypes.POINTER(cf),
                                   ctypes.POINTER(ctypes.c_longlong), ctypes.POINTER(ctypes.c_longlong)]
    lib.apb_layer_info.restype = ci
    lib.apb_layer_export.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.apb_layer_export.restype = ci
    lib.apb_layer_export_steps.argtypes = [vp, ctypes.POINTER(ctypes.c_longlong * 4), vp, vp, vp, vp, vp, vp]
    lib.apb_layer_export_steps.restype = ci
    lib.apb_layer_free.argtypes = [vp]
    lib.apb_layer_free.restype = None
    lib.apb_acts_bytes.argtypes = [ci, ci, ci]
    lib.apb_acts_bytes.restype = ctypes.c_size_t
    lib.apb_quantize_acts.argtypes = [vp, ci, ci, ci, cf, vp, vp]
    lib.apb_quantize_acts.restype = ci
    lib.apb_forward.argtypes = [vp, vp, ci, ci, cf, vp, vp]
    lib.apb_forward.restype = ci
    lib.apb_quantize_forward.argtypes = [vp, vp, ci, ci, cf, vp, vp, vp]
    lib.apb_quantize_forward.restype = ci
    lib.apb_forward_kernel_name.argtypes = [vp, ci, ci]
    lib.apb_forward_kernel_name.restype = ctypes.c_char_p
    lib.apb_quantize_forward_static.argtypes = [vp, vp, ci, ci, cf, vp, vp]
    lib.apb_quantize_forward_static.restype = ci
    lib.apb_quantize_forward_is_one_kernel.argtypes = [vp, ci, ci]
    lib.apb_quantize_forward_is_one_kernel.restype = ci
    lib.apb_forward_requant.argtypes = [vp, vp, ci, ci, cf, vp, vp, ci, cf, vp, vp]
    lib.apb_forward_requant.restype = ci
    lib.apb_forward_conv3x3.argtypes = [vp, vp, ci, ci, ci, ci, ci, cf, vp, ctypes.c_size_t, vp, vp]
    lib.apb_forward_conv3x3.restype = ci
    lib.apb_forward_conv3x3_requant.argtypes = [vp, vp, ci, ci, ci, ci, ci, cf, vp, vp, ci, cf, vp, ctypes.c_size_t, vp, vp]
    lib.apb_forward_conv3x3_requant.restype = ci
    lib.apb_forward_int.argtypes = [vp, vp, ci, ci, vp, vp]
    lib.apb_forward_int.restype = ci
    lib.apb_forward_int_popcount.argtypes = [vp, vp, ci, ci, vp, vp]
    lib.apb_forward_int_popcount.restype = ci
    lib.apb_forward_popcount.argtypes = [vp, vp, ci, ci, cf, vp, vp]
    lib.apb_forward_popcount.restype = ci
    lib.apb_w2_pack.argtypes = [vp, ci, ci, cf, vp, ctypes.POINTER(vp)]
    lib.apb_w2_pack.restype = ci
    lib.apb_w2_export.argtypes = [vp, vp, vp]
    lib.apb_w2_export.restype = ci
    lib.apb_w2_free.argtypes = [vp]
    lib.apb_w2_free.restype = None
    lib.apb_gemm_2_2_int.argtypes = [vp, vp, ci, vp, vp]
    lib.apb_gemm_2_2_int.restype = ci
    lib.apb_gemm_2_2.argtypes = [vp, vp, ci, cf, vp, vp]
    lib.apb_gemm_2_2.restype = ci
    lib.apb_train_workspace_bytes.argtypes = []
    lib.apb_train_workspace_bytes.restype = ctypes.c_size_t
    lib.apb_train_forward.argtypes = [vp, ctypes.c_longlong, cf, cf, vp, vp]
    lib.apb_train_forward.restype = ci
    lib.apb_train_backward.argtypes = [vp, vp, ctypes.c_longlong, cf, cf, vp, vp, vp, vp, vp]
    lib.apb_train_backward.restype = ci
    lib.apb_probe_out_bytes.argtypes = []
    lib.apb_probe_out_bytes.restype = ctypes.c_size_t
    lib.apb_probe_rate.argtypes = [ci, ci, vp, ctypes.POINTER(ctypes.c_double), vp]
    lib.apb_probe_rate.restype = ci
    ll = ctypes.c_longlong
    lib.apb_mx4_bytes.argtypes = [ci, ci]
    lib.apb_mx4_bytes.restype = ctypes.c_size_t
    lib.apb_moe_workspace_bytes.argtypes = [ci, ci, ci]
    lib.apb_moe_workspace_bytes.restype = ctypes.c_size_t
    lib.apb_mx4_linear_scratch_bytes.argtypes = [ci] * 5
    lib.apb_mx4_linear_scratch_bytes.restype = ctypes.c_size_t
    for name in ("apb_mx4_backward_input_workspace_bytes", "apb_mx4_backward_weight_workspace_bytes"):
        getattr(lib, name).argtypes = [ci] * 6
        getattr(lib, name).restype = ctypes.c_size_t
    for name, args in (("apb_mx4_quantize", [vp, ci, ll, ll, ci, vp, ci, ci, vp, vp]),
                       ("apb_mx4_dequantize", [vp, ci, ci, ci, vp, ll, vp]),
                       ("apb_mx4_gemm", [vp, vp, vp, ci, ci, ci, ci, ci, vp, ll, vp]),
                       ("apb_mx4_linear", [vp, ci, ll, ci, vp, vp, vp, ci, ci, ci, ci, vp, ci, vp, ll, vp]),
                       ("apb_mx4_backward_input", [vp, ci, ll, vp, vp, ci, ci, ci, ci, ci, vp, ll, vp, ctypes.c_size_t, vp]),
                       ("apb_mx4_backward_weight", [vp, ci, ll, vp, vp, ci, ci, ci, ci, ci, vp, ll, vp, ctypes.c_size_t, vp]),
                       ("apb_moe_route", [vp, ci, ll, ci, ci, ci, vp, vp, vp, vp, vp, vp, vp]),
                       ("apb_moe_route_backward", [vp, vp, vp, ci, ci, ci, ci, vp, ll, vp]),
                       ("apb_moe_combine", [vp, ci, ll, vp, vp, ci, ci, ci, vp, ll, vp]),
                       ("apb_moe_combine_backward", [vp, ci, ll, vp, ll, vp, vp, ci, ci, ci, vp, ll, vp, vp]),
                       ("apb_mx8_quantize", [vp, ci, ll, ci, ci, vp, vp]),
                       ("apb_mx8_dequantize", [vp, ci, ci, ci, vp, ll, vp]),
                       ("apb_mx4_gated_gemm", [vp, vp, vp, ci, ci, ci, ci, ci, ci, vp, ll, vp, vp]),
                       ("apb_mx4_gated_linear", [vp, ci, ll, ci, vp, vp, vp, ci, ci, ci, ci, ci, vp, ci, vp, ll, vp, vp]),
                       ("apb_gated_forward", [vp, ci, ll, ci, ci, ci, vp, ll, vp, vp]),
                       ("apb_gated_backward", [vp, ci, ll, vp, ci, ll, ci, ci, ci, vp, ll, vp, ll, vp]),
                       ("apb_adapter_parts", [ci] * 4),
                       ("apb_adapter_down", [vp, ci, ll, vp, vp, vp, vp, ci, ci, ci, ci, ci, vp, vp]),
                       ("apb_adapter_up", [vp, ci, vp, ci, vp, vp, ci, ci, ci, ci, ci, vp, ll, vp, ll, vp]),
                       ("apb_adapter_gradient", [vp, ci, vp, ci, ll, vp, vp, ci, ci, ci, ci, ci, vp, vp, ctypes.c_size_t, vp])):
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = ci
    for name, sizes in (("apb_mx8_bytes", 2), ("apb_mx4_gated_linear_scratch_bytes", 6), ("apb_adapter_gradient_workspace_bytes", 5)):
        getattr(lib, name).argtypes = [ci] * sizes
        getattr(lib, name).restype = ctypes.c_size_t
    lib.apb_strerror.argtypes = [ci]
    lib.apb_strerror.restype = ctypes.c_char_p
    lib.apb_last_hip_error.argtypes = []
    lib.apb_last_hip_error.restype = ci
    _lib = lib
    return lib


def strerror(code: int) -> str:
    return load().apb_strerror(int(code)).decode()


def _check(code: int, what: str) -> None:
    if code != APB_OK:
        extra = f" [hipError {load().apb_last_hip_error()}]" if code == APB_ERR_HIP else ""
        raise ApbError(code, what + extra)


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is None:                                   # (the handle alone: a Stream object takes 2.6 us to make)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(stream.cuda_stream)


def _stream_at(stream: Optional[torch.cuda.Stream], first: torch.Tensor, *others: Optional[torch.Tensor]) -> int:
    """_stream for a call with these operands (None: not given), all of which have to be on the current device, like the stream: that
    is where kernels are launched.  (With one device in all, the first one speaks for the others: 0.3 us less of a call's 8.)"""
    here = torch._C._cuda_getDevice()
    if first.get_device() != here:
        raise ValueError("the tensors must be on the current device")
    if _several_devices:
        for t in others:
            if t is not None and t.get_device() != here:
                raise ValueError("the tensors must be on the current device")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(here)
    if stream.device_index != here:
        raise ValueError("the stream must be one of the current device")
    return int(stream.cuda_stream)


def _dev_ptr(t: torch.Tensor, dtype: torch.dtype, name: str) -> int:
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} tensor on the GPU")
    return t.data_ptr()


class ApbLayer:
    """Owner of one opaque apb_layer handle."""

    def __init__(self, handle: int):
        self._h = ctypes.c_void_p(handle)

    @property
    def handle(self) -> ctypes.c_void_p:
        if not self._h:
            raise RuntimeError("layer already freed")
        return self._h

    def info(self) -> dict:
        return apb_layer_info(self)

    def free(self) -> None:
        if self._h:
            load().apb_layer_free(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def apb_compress(W: torch.Tensor, delta: float, alpha: Optional[float] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> ApbLayer:
    """W: [N,K] float32 on the GPU.  alpha=None asks the library for its default scale."""
    if W.dim() != 2:
        raise TypeError("W must be 2-D [N, K]")
    ptr = _dev_ptr(W, torch.float32, "W")
    N, K = W.shape
    out = ctypes.c_void_p(None)
    a = math.nan if alpha is None else float(alpha)
    _check(load().apb_compress(ptr, N, K, float(delta), a, _stream(stream), ctypes.byref(out)), "apb_compress")
    return ApbLayer(out.value)


def apb_layer_info(layer: ApbLayer) -> dict:
    N, K, a = ctypes.c_int(), ctypes.c_int(), ctypes.c_float()
    nnz, bits = ctypes.c_longlong(), ctypes.c_longlong()
    _check(load().apb_layer_info(layer.handle, ctypes.byref(N), ctypes.byref(K), ctypes.byref(a),
                                 ctypes.byref(nnz), ctypes.byref(bits)), "apb_layer_info")
    return {"N": N.value, "K": K.value, "alpha": a.value, "nnz": nnz.value, "mem_bits": bits.value}


def apb_layer_export(layer: ApbLayer, stream: Optional[torch.cuda.Stream] = None) -> dict:
    """Canonical representation as GPU tensors: sign_words uint32-as-int32 [N,Kw], CSR, rowsum."""
    i = apb_layer_info(layer)
    N, K, nnz = i["N"], i["K"], i["nnz"]
    Kw = (K + 31) // 32
    dev = torch.device("cuda", torch.cuda.current_device())
    sign = torch.empty((N, Kw), dtype=torch.int32, device=dev)
    row_ptr = torch.empty(N + 1, dtype=torch.int32, device=dev)
    col = torch.empty(max(nnz, 1), dtype=torch.int32, device=dev)
    val = torch.empty(max(nnz, 1), dtype=torch.float32, device=dev)
    rowsum = torch.empty(N, dtype=torch.int32, device=dev)
    _check(load().apb_layer_export(layer.handle, sign.data_ptr(), row_ptr.data_ptr(), col.data_ptr(),
                                   val.data_ptr(), rowsum.data_ptr(), _stream(stream)), "apb_layer_export")
    return {"sign_words": sign, "row_ptr": row_ptr, "col_idx": col[:nnz], "val": val[:nnz], "rowsum": rowsum,
            **i}


def apb_layer_export_steps(layer: ApbLayer, stream: Optional[torch.cuda.Stream] = None) -> dict:
    """Test hook: the operands of the matrix-core forward kernel, as GPU tensors ("steps": 0 if none were built)."""
    sizes = (ctypes.c_longlong * 4)()
    call, s = load().apb_layer_export_steps, _stream(stream)
    _check(call(layer.handle, ctypes.byref(sizes), None, None, None, None, None, s), "apb_layer_export_steps")
    steps, windows, unit, words = sizes
    if steps == 0:
        return {"steps": 0}
    tiles = 2 * ((apb_layer_info(layer)["N"] + 31) // 32)
    dev = torch.device("cuda", torch.cuda.current_device())
    out = {"first": torch.empty(tiles + 1, dtype=torch.int32, device=dev),
           "count": torch.empty(2 * tiles * windows, dtype=torch.uint8, device=dev),
           "step": torch.empty(((steps + 8), 1408), dtype=torch.uint8, device=dev),
           "valsum": torch.empty(16 * tiles, dtype=torch.float64, device=dev),
           "sign": torch.empty(words, dtype=torch.int32, device=dev)}
    _check(call(layer.handle, ctypes.byref(sizes), *(t.data_ptr() for t in out.values()), s), "apb_layer_export_steps")
    return {"steps": steps, "windows": windows, "unit": unit, **out}


def apb_acts_bytes(K: int, M: int, bits: int) -> int:
    return int(load().apb_acts_bytes(int(K), int(M), int(bits)))


def alloc_packed(K: int, M: int, bits: int, device=None) -> torch.Tensor:
    nbytes = apb_acts_bytes(K, M, bits)
    if nbytes == 0:
        raise ApbError(APB_ERR_SHAPE if bits in (1, 2) else APB_ERR_BITS, "apb_acts_bytes")
    dev = device if device is not None else torch.device("cuda", torch.cuda.current_device())
    return torch.empty(nbytes // 4, dtype=torch.int32, device=dev)


def apb_quantize_acts(X: torch.Tensor, bits: int, step: float, packed: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """X: [K,M] float32 on the GPU -> packed int32 buffer (planes + column sums)."""
    if X.dim() != 2:
        raise TypeError("X must be 2-D [K, M]")
    ptr = _dev_ptr(X, torch.float32, "X")
    K, M = X.shape
    if packed is None:
        packed = alloc_packed(K, M, bits, X.device)
    elif packed.numel() * packed.element_size() < apb_acts_bytes(K, M, bits):
        raise ValueError("packed buffer too small")
    _check(load().apb_quantize_acts(ptr, K, M, int(bits), float(step), _dev_ptr(packed, torch.int32, "packed"),
                                    _stream(stream)), "apb_quantize_acts")
    return packed


def _check_packed(layer: ApbLayer, packed: torch.Tensor, M: int, bits: int) -> Tuple[int, int]:
    i = apb_layer_info(layer)
    need = apb_acts_bytes(i["K"], M, bits)
    if need and packed.numel() * packed.element_size() < need:
        raise ValueError("packed buffer smaller than apb_acts_bytes(K, M, bits)")
    return i["N"], i["K"]


def apb_forward(layer: ApbLayer, packed: torch.Tensor, M: int, bits: int, step: float,
                Y: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    N, _ = _check_packed(layer, packed, M, bits)
    if Y is None:
        Y = torch.empty((N, M), dtype=torch.float32, device=packed.device)
    elif tuple(Y.shape) != (N, M):
        raise ValueError("Y must be [N, M]")
    _check(load().apb_forward(layer.handle, _dev_ptr(packed, torch.int32, "packed"), int(M), int(bits),
                              float(step), _dev_ptr(Y, torch.float32, "Y"), _stream(stream)), "apb_forward")
    return Y


def apb_quantize_forward(layer: ApbLayer, X: torch.Tensor, bits: int, step: float, packed: Optional[torch.Tensor] = None,
                         Y: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """apb_quantize_acts + apb_forward in one call; `packed` is scratch."""
    if X.dim() != 2:
        raise TypeError("X must be 2-D [K, M]")
    K, M = X.shape
    if packed is None:
        packed = alloc_packed(K, M, bits, X.device)
    N, _ = _check_packed(layer, packed, M, bits)
    if apb_layer_info(layer)["K"] != K:
        raise ValueError("X must have the layer's K rows")
    if Y is None:
        Y = torch.empty((N, M), dtype=torch.float32, device=X.device)
    elif tuple(Y.shape) != (N, M):
        raise ValueError("Y must be [N, M]")
    _check(load().apb_quantize_forward(layer.handle, _dev_ptr(X, torch.float32, "X"), int(M), int(bits), float(step),
                                       _dev_ptr(packed, torch.int32, "packed"), _dev_ptr(Y, torch.float32, "Y"),
                                       _stream(stream)), "apb_quantize_forward")
    return Y


def apb_forward_kernel_name(layer: ApbLayer, M: int, bits: int) -> str:
    return load().apb_forward_kernel_name(layer.handle, int(M), int(bits)).decode()


def apb_quantize_forward_static(layer: ApbLayer, X: torch.Tensor, bits: int, step: float, Y: torch.Tensor,
                                stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """apb_quantize_forward through the library's static scratch array; allocates nothing (Y is the caller's)."""
    if X.dim() != 2:
        raise TypeError("X must be 2-D [K, M]")
    K, M = X.shape
    i = apb_layer_info(layer)
    if i["K"] != K:
        raise ValueError("X must have the layer's K rows")
    if tuple(Y.shape) != (i["N"], M):
        raise ValueError("Y must be [N, M]")
    _check(load().apb_quantize_forward_static(layer.handle, _dev_ptr(X, torch.float32, "X"), int(M), int(bits),
                                              float(step), _dev_ptr(Y, torch.float32, "Y"), _stream(stream)),
           "apb_quantize_forward_static")
    return Y


def apb_quantize_forward_is_one_kernel(layer: ApbLayer, M: int, bits: int) -> bool:
    return bool(load().apb_quantize_forward_is_one_kernel(layer.handle, int(M), int(bits)))


def apb_forward_requant(layer: ApbLayer, packed: torch.Tensor, M: int, bits: int, step: float, bits_out: int,
                        step_out: float, scale: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None,
                        packed_out: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The layer's output, quantized for the next layer and packed (its K = this layer's N)."""
    N, _ = _check_packed(layer, packed, M, bits)
    if (scale is None) != (shift is None):
        raise ValueError("scale and shift go together")
    for name, t in (("scale", scale), ("shift", shift)):
        if t is not None and t.numel() != N:
            raise ValueError(f"{name} must hold N floats")
    if packed_out is None:
        packed_out = alloc_packed(N, M, bits_out, packed.device)
    elif packed_out.numel() * packed_out.element_size() < apb_acts_bytes(N, M, bits_out):
        raise ValueError("packed_out smaller than apb_acts_bytes(N, M, bits_out)")
    _check(load().apb_forward_requant(layer.handle, _dev_ptr(packed, torch.int32, "packed"), int(M), int(bits),
                                      float(step), None if scale is None else _dev_ptr(scale, torch.float32, "scale"),
                                      None if shift is None else _dev_ptr(shift, torch.float32, "shift"),
                                      int(bits_out), float(step_out), _dev_ptr(packed_out, torch.int32, "packed_out"),
                                      _stream(stream)), "apb_forward_requant")
    return packed_out


def _workspace(t: Optional[torch.Tensor]):
    """(pointer, bytes) of an optional scratch tensor."""
    if t is None:
        return None, 0
    return _dev_ptr(t, torch.int32, "workspace"), t.numel() * t.element_size()


def _check_fmap(layer: ApbLayer, fmap: torch.Tensor, B: int, H: int, W: int, bits: int, stride: int) -> Tuple[int, int]:
    """(N, output pixels B*Ho*Wo) after checking the size of the input map's buffer."""
    i = apb_layer_info(layer)
    if i["K"] % 9:
        raise ValueError("the layer's K is not 9 * C")
    if stride not in (1, 2):
        raise ValueError("stride must be 1 or 2")
    P = int(B) * int(H) * int(W)
    need = apb_acts_bytes(i["K"] // 9, P, bits)
    if need and fmap.numel() * fmap.element_size() < need:
        raise ValueError("fmap smaller than apb_acts_bytes(C, B*H*W, bits)")
    return i["N"], int(B) * ((int(H) - 1) // stride + 1) * ((int(W) - 1) // stride + 1)


def apb_forward_conv3x3(layer: ApbLayer, fmap: torch.Tensor, B: int, H: int, W: int, bits: int, step: float,
                        Y: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
                        stride: int = 1, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """3x3 convolution (padding 1) over a packed feature map [C, B*H*W]; Y is [N, B*Ho*Wo].  `workspace`: an
    optional int32 scratch tensor (see the header)."""
    N, P = _check_fmap(layer, fmap, B, H, W, bits, stride)
    if Y is None:
        Y = torch.empty((N, P), dtype=torch.float32, device=fmap.device)
    elif tuple(Y.shape) != (N, P):
        raise ValueError("Y must be [N, B*Ho*Wo]")
    _check(load().apb_forward_conv3x3(layer.handle, _dev_ptr(fmap, torch.int32, "fmap"), int(B), int(H), int(W), int(stride),
                                      int(bits), float(step), *_workspace(workspace), _dev_ptr(Y, torch.float32, "Y"),
                                      _stream(stream)),
           "apb_forward_conv3x3")
    return Y


def apb_forward_conv3x3_requant(layer: ApbLayer, fmap: torch.Tensor, B: int, H: int, W: int, bits: int, step: float,
                                bits_out: int, step_out: float, scale: Optional[torch.Tensor] = None,
                                shift: Optional[torch.Tensor] = None, fmap_out: Optional[torch.Tensor] = None,
                                stream: Optional[torch.cuda.Stream] = None, stride: int = 1,
                                workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    N, P = _check_fmap(layer, fmap, B, H, W, bits, stride)
    if (scale is None) != (shift is None):
        raise ValueError("scale and shift go together")
    for name, t in (("scale", scale), ("shift", shift)):
        if t is not None and t.numel() != N:
            raise ValueError(f"{name} must hold N floats")
    if fmap_out is None:
        fmap_out = alloc_packed(N, P, bits_out, fmap.device)
    elif fmap_out.numel() * fmap_out.element_size() < apb_acts_bytes(N, P, bits_out):
        raise ValueError("fmap_out smaller than apb_acts_bytes(N, B*Ho*Wo, bits_out)")
    _check(load().apb_forward_conv3x3_requant(
        layer.handle, _dev_ptr(fmap, torch.int32, "fmap"), int(B), int(H), int(W), int(stride), int(bits), float(step),
        None if scale is None else _dev_ptr(scale, torch.float32, "scale"),
        None if shift is None else _dev_ptr(shift, torch.float32, "shift"), int(bits_out), float(step_out),
        *_workspace(workspace), _dev_ptr(fmap_out, torch.int32, "fmap_out"), _stream(stream)), "apb_forward_conv3x3_requant")
    return fmap_out


def apb_forward_int(layer: ApbLayer, packed: torch.Tensor, M: int, bits: int,
                    D: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    N, _ = _check_packed(layer, packed, M, bits)
    if D is None:
        D = torch.empty((N, M), dtype=torch.int32, device=packed.device)
    elif tuple(D.shape) != (N, M):
        raise ValueError("D must be [N, M]")
    _check(load().apb_forward_int(layer.handle, _dev_ptr(packed, torch.int32, "packed"), int(M), int(bits),
                                  _dev_ptr(D, torch.int32, "D"), _stream(stream)), "apb_forward_int")
    return D


def apb_forward_int_popcount(layer: ApbLayer, packed: torch.Tensor, M: int, bits: int,
                             D: Optional[torch.Tensor] = None,
                             stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    N, _ = _check_packed(layer, packed, M, bits)
    if D is None:
        D = torch.empty((N, M), dtype=torch.int32, device=packed.device)
    elif tuple(D.shape) != (N, M):
        raise ValueError("D must be [N, M]")
    _check(load().apb_forward_int_popcount(layer.handle, _dev_ptr(packed, torch.int32, "packed"), int(M), int(bits),
                                           _dev_ptr(D, torch.int32, "D"), _stream(stream)),
           "apb_forward_int_popcount")
    return D


def apb_forward_popcount(layer: ApbLayer, packed: torch.Tensor, M: int, bits: int, step: float,
                         Y: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    N, _ = _check_packed(layer, packed, M, bits)
    if Y is None:
        Y = torch.empty((N, M), dtype=torch.float32, device=packed.device)
    elif tuple(Y.shape) != (N, M):
        raise ValueError("Y must be [N, M]")
    _check(load().apb_forward_popcount(layer.handle, _dev_ptr(packed, torch.int32, "packed"), int(M), int(bits),
                                       float(step), _dev_ptr(Y, torch.float32, "Y"), _stream(stream)),
           "apb_forward_popcount")
    return Y


# ----------------------------------------------------------------------------- 2/2 routine

class ApbW2:
    """Owner of an apb_w2 handle (packed 2-bit weights)."""

    def __init__(self, handle: int, N: int, K: int):
        self._h = ctypes.c_void_p(handle)
        self.N, self.K = N, K

    @property
    def handle(self) -> ctypes.c_void_p:
        if not self._h:
            raise RuntimeError("weights already freed")
        return self._h

    def free(self) -> None:
        if self._h:
            load().apb_w2_free(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def apb_w2_pack(W: torch.Tensor, step_w: float, stream: Optional[torch.cuda.Stream] = None) -> ApbW2:
    if W.dim() != 2:
        raise ValueError("W must be [N, K]")
    ptr = _dev_ptr(W, torch.float32, "W")
    N, K = int(W.shape[0]), int(W.shape[1])
    out = ctypes.c_void_p(None)
    _check(load().apb_w2_pack(ptr, N, K, float(step_w), _stream(stream), ctypes.byref(out)), "apb_w2_pack")
    return ApbW2(out.value, N, K)


def apb_w2_export(w2: ApbW2, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """int32 view of the canonical planes, shape [2, N, ceil(K/32)]."""
    Kw = (w2.K + 31) // 32
    planes = torch.empty((2, w2.N, Kw), dtype=torch.int32, device="cuda")
    _check(load().apb_w2_export(w2.handle, planes.data_ptr(), _stream(stream)), "apb_w2_export")
    return planes


def _check_packed_w2(w2: ApbW2, packed: torch.Tensor, M: int) -> None:
    need = apb_acts_bytes(w2.K, M, 2)
    if need == 0:
        raise ValueError("bad K, M")
    if packed.numel() * packed.element_size() < need:
        raise ValueError("packed buffer smaller than apb_acts_bytes(K, M, 2)")


def apb_gemm_2_2_int(w2: ApbW2, packed: torch.Tensor, M: int, D: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    _check_packed_w2(w2, packed, M)
    if D is None:
        D = torch.empty((w2.N, M), dtype=torch.int32, device=packed.device)
    elif tuple(D.shape) != (w2.N, M):
        raise ValueError("D must be [N, M]")
    _check(load().apb_gemm_2_2_int(w2.handle, _dev_ptr(packed, torch.int32, "packed"), int(M),
                                   _dev_ptr(D, torch.int32, "D"), _stream(stream)), "apb_gemm_2_2_int")
    return D


def apb_gemm_2_2(w2: ApbW2, packed: torch.Tensor, M: int, step_a: float, Y: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    _check_packed_w2(w2, packed, M)
    if Y is None:
        Y = torch.empty((w2.N, M), dtype=torch.float32, device=packed.device)
    elif tuple(Y.shape) != (w2.N, M):
        raise ValueError("Y must be [N, M]")
    _check(load().apb_gemm_2_2(w2.handle, _dev_ptr(packed, torch.int32, "packed"), int(M), float(step_a),
                               _dev_ptr(Y, torch.float32, "Y"), _stream(stream)), "apb_gemm_2_2")
    return Y


# ----------------------------------------------------------------------------- instruction-rate probes

PROBES = {"mfma_fp4": 0, "mfma_i8": 1, "and_bcnt": 2, "fma_f64": 3, "lds_u8": 4, "lds_b128": 5, "mfma_fp4_lds": 6,
          "mfma_fp4_lds_barrier": 7, "mfma_fp4_lds_barrier_valu": 8}


def apb_probe_out_bytes() -> int:
    return int(load().apb_probe_out_bytes())


def apb_probe_rate(kind: int, iters: int, out: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> float:
    """Launch one probe; returns the work of the launch (flops or lane operations)."""
    if out.numel() * out.element_size() < apb_probe_out_bytes():
        raise ValueError("out smaller than apb_probe_out_bytes()")
    work = ctypes.c_double()
    _check(load().apb_probe_rate(int(kind), int(iters), out.data_ptr(), ctypes.byref(work), _stream(stream)),
           "apb_probe_rate")
    return work.value


# ----------------------------------------------------------------------------- training-side operators

def apb_train_workspace_bytes() -> int:
    return int(load().apb_train_workspace_bytes())


def apb_train_forward(W: torch.Tensor, alpha: float, delta: float, out: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """APB(w) element-wise on the latent weights (any shape, contiguous float32)."""
    ptr = _dev_ptr(W, torch.float32, "W")
    if out is None:
        out = torch.empty_like(W)
    elif out.shape != W.shape:
        raise ValueError("out must have W's shape")
    _check(load().apb_train_forward(ptr, W.numel(), float(alpha), float(delta), _dev_ptr(out, torch.float32, "out"),
                                    _stream(stream)), "apb_train_forward")
    return out


def apb_train_backward(W: torch.Tensor, G: torch.Tensor, alpha: float, delta: float, want_grad_w: bool = True,
                       grad_w: Optional[torch.Tensor] = None, sums: Optional[torch.Tensor] = None,
                       count: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None):
    """Returns (grad_w or None, sums [grad_alpha, grad_delta] float64 on the GPU, count int64 on the GPU)."""
    if W.shape != G.shape:
        raise ValueError("G must have W's shape")
    if want_grad_w and grad_w is None:
        grad_w = torch.empty_like(G)
    if sums is None:
        sums = torch.empty(2, dtype=torch.float64, device=W.device)
    if count is None:
        count = torch.empty(1, dtype=torch.int64, device=W.device)
    if workspace is None:
        workspace = torch.empty(apb_train_workspace_bytes() // 8, dtype=torch.float64, device=W.device)
    elif workspace.numel() * workspace.element_size() < apb_train_workspace_bytes():
        raise ValueError("workspace smaller than apb_train_workspace_bytes()")
    _check(load().apb_train_backward(_dev_ptr(W, torch.float32, "W"), _dev_ptr(G, torch.float32, "G"), W.numel(),
                                     float(alpha), float(delta),
                                     None if grad_w is None else _dev_ptr(grad_w, torch.float32, "grad_w"),
                                     sums.data_ptr(), count.data_ptr(), workspace.data_ptr(), _stream(stream)),
           "apb_train_backward")
    return grad_w, sums, count


# ----------------------------------------------------------------------------- microscaled 4-bit matrices

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}      # apb_type


def _type(dtype: torch.dtype) -> int:
    t = _TYPES.get(dtype)
    if t is None:
        raise TypeError("element type must be float32, bfloat16 or float16")
    return t


# (The C entry points count in int, and ctypes passes the low 32 bits of what is larger: such sizes end here.)
def _matrix(t: torch.Tensor, name: str) -> Tuple[int, int, int]:
    """(pointer, apb_type, row stride) of a 2-D float matrix whose rows are contiguous."""
    if not t.is_cuda or t.dim() != 2:
        raise TypeError(f"{name} must be a 2-D tensor on the GPU")
    rows, cols = t.shape
    if (rows | cols) >> 31:
        raise ApbError(APB_ERR_SHAPE, name)
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise TypeError(f"the rows of {name} must be contiguous")
    return t.data_ptr(), _type(t.dtype), ld if rows > 1 else max(cols, ld)


def _new(like: torch.Tensor, shape, dtype: torch.dtype, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """Memory beside `like` for a call on `stream`: that stream's own, so nothing under way on another one has it, before or after."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _result(t: Optional[torch.Tensor], shape: Tuple[int, int], dtype: torch.dtype, like: torch.Tensor, name: str,
            stream: Optional[torch.cuda.Stream]):
    """(tensor, pointer, apb_type, row stride) of an output: `t`, or a new one beside `like`."""
    if t is None:
        if (shape[0] | shape[1]) >> 31:                                   # (negative ones as well)
            raise ApbError(APB_ERR_SHAPE, name)
        t = _new(like, shape, dtype, stream)
        return t, t.data_ptr(), _type(dtype), shape[1]
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}")
    return (t, *_matrix(t, name))


def _array(t: Optional[torch.Tensor], dtype: torch.dtype, count: Optional[int], name: str) -> Optional[int]:
    """Pointer of a contiguous array of `count` entries, None for None."""
    if t is None:
        return None
    if count is not None and t.numel() != count:
        raise ValueError(f"{name} must hold {count} entries")
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} tensor on the GPU")
    return t.data_ptr()


def apb_mx4_bytes(rows: int, K: int) -> int:
    return int(load().apb_mx4_bytes(int(rows), int(K)))


def alloc_mx4(rows: int, K: int, device=None) -> torch.Tensor:
    """Memory for a 4-bit matrix of `rows` rows of K values (uint8, see the header for the layout)."""
    nbytes = apb_mx4_bytes(rows, K)
    if nbytes == 0:
        raise ApbError(APB_ERR_SHAPE, "apb_mx4_bytes")
    dev = device if device is not None else torch.device("cuda", torch.cuda.current_device())
    return torch.empty(nbytes, dtype=torch.uint8, device=dev)


def _new_mx4(like: torch.Tensor, rows: int, K: int, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    nbytes = apb_mx4_bytes(rows, K)
    if nbytes == 0:
        raise ApbError(APB_ERR_SHAPE, "apb_mx4_bytes")
    return _new(like, nbytes, torch.uint8, stream)


def _mx4_ptr(mx: torch.Tensor, rows: int, K: int, name: str) -> int:
    # (what apb_mx4_bytes says; the library refuses the sizes it has no answer for)
    if mx.numel() < rows * ((K + 255) // 256) * 136:
        raise ValueError(f"{name} smaller than apb_mx4_bytes({rows}, {K})")
    return _array(mx, torch.uint8, None, name)


def _experts(offsets: Optional[torch.Tensor]) -> Tuple[Optional[int], int]:
    """(pointer, number of groups) of the offsets; (None, 1) without."""
    if offsets is None:
        return None, 1
    E = offsets.numel() - 1
    if E < 1:
        raise ValueError("offsets must hold E + 1 int32")
    if E >> 31:
        raise ApbError(APB_ERR_SHAPE, "offsets")
    return _array(offsets, torch.int32, None, "offsets"), E


def apb_mx4_quantize(X: torch.Tensor, mx: Optional[torch.Tensor] = None, rows_from: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """X: [rows, K] on the GPU, any strides (X.t() of a K x M matrix as well) -> its 4-bit form.  rows_from: int32 [rows],
    the rows of X to take."""
    if X.dim() != 2 or not X.is_cuda:
        raise TypeError("X must be a 2-D tensor on the GPU")
    rows_in, K = X.shape
    rows = rows_in if rows_from is None else rows_from.numel()
    if mx is None:
        mx = _new_mx4(X, rows, K, stream)
    _check(load().apb_mx4_quantize(X.data_ptr(), _type(X.dtype), X.stride(0), 1 if K == 1 else X.stride(1), rows_in,
                                   _array(rows_from, torch.int32, rows, "rows_from"), rows, K, _mx4_ptr(mx, rows, K, "mx"), _stream(stream)),
           "apb_mx4_quantize")
    return mx


def apb_mx4_dequantize(mx: torch.Tensor, rows: int, K: int, dtype: torch.dtype = torch.float32,
                       X: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    X, ptr, t, ld = _result(X, (rows, K), dtype, mx, "X", stream)
    _check(load().apb_mx4_dequantize(_mx4_ptr(mx, rows, K, "mx"), int(rows), int(K), t, ptr, ld, _stream(stream)),
           "apb_mx4_dequantize")
    return X


def apb_mx4_gemm(A: torch.Tensor, B: torch.Tensor, M: int, N: int, K: int, dtype: torch.dtype = torch.float32,
                 Y: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Y[M, N] = A^ B^T of two 4-bit matrices; with offsets (int32 [E+1]) the rows of A are grouped by expert and B holds
    E*N rows."""
    off, E = _experts(offsets)
    Y, ptr, t, ld = _result(Y, (M, N), dtype, A, "Y", stream)
    _check(load().apb_mx4_gemm(_mx4_ptr(A, M, K, "A"), _mx4_ptr(B, E * N, K, "B"), off, E, int(M), int(N), int(K), t, ptr, ld,
                               _stream(stream)), "apb_mx4_gemm")
    return Y


def apb_mx4_linear_scratch_bytes(grouped: bool, E: int, M: int, N: int, K: int) -> int:
    """Bytes of scratch that apb_mx4_linear uses: 0 where it runs as one kernel."""
    return int(load().apb_mx4_linear_scratch_bytes(int(grouped), E, M, N, K))


def apb_mx4_linear(X: torch.Tensor, W: torch.Tensor, N: int, dtype: Optional[torch.dtype] = None,
                   Y: Optional[torch.Tensor] = None, rows_from: Optional[torch.Tensor] = None,
                   offsets: Optional[torch.Tensor] = None, scratch: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """apb_mx4_quantize of X [rows_in, K] + apb_mx4_gemm with the 4-bit weights W in one call; Y has X's type by default."""
    xp, xt, ldx = _matrix(X, "X")
    rows_in, K = X.shape
    M = rows_in if rows_from is None else rows_from.numel()
    off, E = _experts(offsets)
    lib, wp = load(), _mx4_ptr(W, E * N, K, "W")
    if scratch is not None:
        sp = _array(scratch, torch.uint8, None, "scratch")
        if scratch.numel() < M * ((K + 255) // 256) * 136:            # (whole 4-bit matrices are always enough: nothing is asked)
            if scratch.numel() < lib.apb_mx4_linear_scratch_bytes(off is not None, E, M, N, K):
                raise ValueError("scratch smaller than apb_mx4_linear_scratch_bytes(...)")
            sp = wp                                                   # (none needed: not touched, but not NULL)
    else:
        need = lib.apb_mx4_linear_scratch_bytes(off is not None, E, M, N, K)
        scratch = _new(X, need, torch.uint8, stream) if need else None
        sp = scratch.data_ptr() if need else wp
    Y, yp, yt, ldy = _result(Y, (M, N), dtype or X.dtype, X, "Y", stream)
    _check(lib.apb_mx4_linear(xp, xt, ldx, rows_in, _array(rows_from, torch.int32, M, "rows_from"), wp, off, E, M, int(N), K, sp, yt, yp,
                              ldy, _stream(stream)), "apb_mx4_linear")
    return Y


def apb_mx4_backward_input_workspace_bytes(dtype: torch.dtype, grouped: bool, E: int, M: int, N: int, K: int) -> int:
    """Bytes of scratch that apb_mx4_backward_input has a use for, with a gradient of type dtype."""
    return int(load().apb_mx4_backward_input_workspace_bytes(_type(dtype), int(grouped), E, M, N, K))


def apb_mx4_backward_weight_workspace_bytes(dtype: torch.dtype, grouped: bool, E: int, M: int, N: int, K: int) -> int:
    return int(load().apb_mx4_backward_weight_workspace_bytes(_type(dtype), int(grouped), E, M, N, K))


def _scratch(given: Optional[torch.Tensor], need: int, like: torch.Tensor, stream: Optional[torch.cuda.Stream]):
    """(tensor to keep, pointer, bytes) of an optional workspace; a new one where none is given and one is of use."""
    if given is None:
        if need == 0:
            return None, None, 0
        given = _new(like, need, torch.uint8, stream)
    if not given.is_cuda or not given.is_contiguous():
        raise TypeError("workspace must be a contiguous tensor on the GPU")
    return given, given.data_ptr(), given.numel() * given.element_size()


def apb_mx4_backward_input(G: torch.Tensor, W: torch.Tensor, K: int, dtype: Optional[torch.dtype] = None,
                           dX: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """dX[M, K] = G W^ for the gradient G [M, N] of the product with the 4-bit weights W; dX has G's type by default."""
    gp, gt, ldg = _matrix(G, "G")
    M, N = G.shape
    off, E = _experts(offsets)
    wp = _mx4_ptr(W, E * N, K, "W")
    dX, xp, xt, ldx = _result(dX, (M, K), dtype or G.dtype, G, "dX", stream)
    lib = load()
    keep, sp, sb = _scratch(workspace, lib.apb_mx4_backward_input_workspace_bytes(gt, off is not None, E, M, N, K), G, stream)
    _check(lib.apb_mx4_backward_input(gp, gt, ldg, wp, off, E, M, N, K, xt, xp, ldx, sp, sb, _stream(stream)), "apb_mx4_backward_input")
    return dX


def apb_mx4_backward_weight(G: torch.Tensor, X: torch.Tensor, K: int, dtype: torch.dtype = torch.float32,
                            dW: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None,
                            workspace: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """dW[E*N, K] = G^T X^ (per expert with offsets) for the 4-bit activations X of the product."""
    gp, gt, ldg = _matrix(G, "G")
    M, N = G.shape
    off, E = _experts(offsets)
    xp = _mx4_ptr(X, M, K, "X")
    dW, wp, wt, ldw = _result(dW, (E * N, K), dtype, G, "dW", stream)
    lib = load()
    keep, sp, sb = _scratch(workspace, lib.apb_mx4_backward_weight_workspace_bytes(gt, off is not None, E, M, N, K), G, stream)
    _check(lib.apb_mx4_backward_weight(gp, gt, ldg, xp, off, E, M, N, K, wt, wp, ldw, sp, sb, _stream(stream)), "apb_mx4_backward_weight")
    return dW


# ----------------------------------------------------------------------------- routing tokens to experts

def apb_moe_workspace_bytes(T: int, E: int, k: int) -> int:
    return int(load().apb_moe_workspace_bytes(int(T), int(E), int(k)))


def alloc_moe_workspace(T: int, E: int, k: int, device=None) -> torch.Tensor:
    nbytes = apb_moe_workspace_bytes(T, E, k)
    if nbytes == 0:
        raise ApbError(APB_ERR_SHAPE, "apb_moe_workspace_bytes")
    dev = device if device is not None else torch.device("cuda", torch.cuda.current_device())
    return torch.empty((nbytes + 3) // 4, dtype=torch.int32, device=dev)


def apb_moe_route(logits: torch.Tensor, k: int, workspace: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> dict:
    """logits [T, E] -> expert int32 [T, k], weight float32 [T, k], offsets int32 [E+1], row_token int32 [T*k],
    slot_row int32 [T, k] (see the header)."""
    ptr, t, ld = _matrix(logits, "logits")
    T, E = logits.shape
    need = apb_moe_workspace_bytes(T, E, k)
    if need == 0:
        raise ApbError(APB_ERR_SHAPE, "apb_moe_route")
    if workspace is not None and workspace.numel() * workspace.element_size() < need:
        raise ValueError("workspace smaller than apb_moe_workspace_bytes(T, E, k)")
    # (one piece of memory for all whole numbers: making one takes half as long as launching a kernel)
    ints, slots = torch.int32, T * k
    expert, slot_row, row_token, offsets, made = _new(logits, 3 * slots + E + 1 + (need + 3) // 4, ints, stream).split_with_sizes(
        (slots, slots, slots, E + 1, (need + 3) // 4))
    weight = _new(logits, (T, k), torch.float32, stream)
    _check(load().apb_moe_route(ptr, t, ld, T, E, k, expert.data_ptr(), weight.data_ptr(), offsets.data_ptr(),
                                row_token.data_ptr(), slot_row.data_ptr(),
                                made.data_ptr() if workspace is None else _array(workspace, ints, None, "workspace"),
                                _stream(stream)), "apb_moe_route")
    expert, slot_row = expert.view(T, k), slot_row.view(T, k)
    return {"expert": expert, "weight": weight, "offsets": offsets, "row_token": row_token, "slot_row": slot_row}


def apb_moe_route_backward(expert: torch.Tensor, weight: torch.Tensor, dweight: torch.Tensor, E: int,
                           dtype: torch.dtype = torch.float32, dlogits: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    if expert.dim() != 2:
        raise ValueError("expert must be [T, k]")
    T, k = expert.shape
    dlogits, ptr, t, ld = _result(dlogits, (T, E), dtype, expert, "dlogits", stream)
    _check(load().apb_moe_route_backward(_array(expert, torch.int32, T * k, "expert"), _array(weight, torch.float32, T * k, "weight"),
                                         _array(dweight, torch.float32, T * k, "dweight"), T, int(E), k, t, ptr, ld, _stream(stream)),
           "apb_moe_route_backward")
    return dlogits


def _slots(slot_row: torch.Tensor, Z: Optional[torch.Tensor], name: str) -> Tuple[int, int]:
    if slot_row.dim() != 2:
        raise ValueError("slot_row must be [T, k]")
    T, k = slot_row.shape
    if Z is not None and Z.shape[0] != T * k:
        raise ValueError(f"{name} must have T*k rows")
    return T, k


def apb_moe_combine(Z: torch.Tensor, slot_row: torch.Tensor, weight: Optional[torch.Tensor] = None,
                    Y: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Y[t] = sum_j weight[t, j] * Z[slot_row[t, j]]; weight None: all 1.  Y has Z's type."""
    T, k = _slots(slot_row, Z, "Z")
    zp, zt, ldz = _matrix(Z, "Z")
    N = Z.shape[1]
    Y, yp, yt, ldy = _result(Y, (T, N), Z.dtype, Z, "Y", stream)
    if yt != zt:
        raise TypeError("Y must have Z's type")
    _check(load().apb_moe_combine(zp, zt, ldz, _array(slot_row, torch.int32, T * k, "slot_row"), _array(weight, torch.float32, T * k, "weight"), T, k, N, yp,
                                  ldy, _stream(stream)), "apb_moe_combine")
    return Y


def apb_moe_combine_backward(dY: torch.Tensor, Z: Optional[torch.Tensor], slot_row: torch.Tensor,
                             weight: Optional[torch.Tensor] = None, dZ: Optional[torch.Tensor] = None,
                             stream: Optional[torch.cuda.Stream] = None):
    """(dZ [T*k, N], dweight float32 [T, k]); Z None: only dZ is computed, dweight is None."""
    T, k = _slots(slot_row, Z, "Z")
    gp, gt, ldg = _matrix(dY, "dY")
    N = dY.shape[1]
    if dY.shape[0] != T:
        raise ValueError("dY must have T rows")
    zp, ldz, dweight = None, N, None
    if Z is not None:
        zp, zt, ldz = _matrix(Z, "Z")
        if Z.shape[1] != N or zt != gt:
            raise ValueError("Z must have dY's columns and type")
        dweight = _new(slot_row, (T, k), torch.float32, stream)
    dZ, dp, dt, lddz = _result(dZ, (T * k, N), dY.dtype, dY, "dZ", stream)
    if dt != gt:
        raise TypeError("dZ must have dY's type")
    _check(load().apb_moe_combine_backward(gp, gt, ldg, zp, ldz, _array(slot_row, torch.int32, T * k, "slot_row"),
                                           _array(weight, torch.float32, T * k, "weight"), T, k, N, dp, lddz,
                                           None if dweight is None else dweight.data_ptr(), _stream(stream)),
           "apb_moe_combine_backward")
    return dZ, dweight


# ----------------------------------------------------------------------------- 8-bit activation checkpoints

_MX8 = 3                                                              # APB_MX8


def apb_mx8_bytes(rows: int, K: int) -> int:
    rows, K = int(rows), int(K)
    return 0 if (rows | K) >> 31 else int(load().apb_mx8_bytes(rows, K))


def alloc_mx8(rows: int, K: int, device=None) -> torch.Tensor:
    """Memory for an 8-bit matrix of `rows` rows of K values (uint8, see the header for the layout)."""
    blocks = (K + 31) // 32                                           # (apb_mx8_bytes without the call)
    if rows <= 0 or K <= 0 or K > 1 << 22 or rows * blocks > (1 << 30) - 64:
        raise ApbError(APB_ERR_SHAPE, "apb_mx8_bytes")
    return torch.empty(rows * blocks * 33, dtype=torch.uint8, device="cuda" if device is None else device)


def _mx8_ptr(mx8: Optional[torch.Tensor], rows: int, K: int, name: str) -> Optional[int]:
    if mx8 is None:
        return None
    if mx8.numel() < rows * ((K + 31) // 32) * 33:                    # (as _mx4_ptr)
        raise ValueError(f"{name} smaller than apb_mx8_bytes({rows}, {K})")
    return _array(mx8, torch.uint8, None, name)


def apb_mx8_quantize(X: torch.Tensor, mx8: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """X [rows, K] -> its 8-bit form."""
    ptr, t, ld = _matrix(X, "X")
    rows, K = X.shape
    if mx8 is None:
        nbytes = apb_mx8_bytes(rows, K)
        if nbytes == 0:
            raise ApbError(APB_ERR_SHAPE, "apb_mx8_bytes")
        mx8 = _new(X, nbytes, torch.uint8, stream)
    _check(load().apb_mx8_quantize(ptr, t, ld, rows, K, _mx8_ptr(mx8, rows, K, "mx8"), _stream_at(stream, X, mx8)), "apb_mx8_quantize")
    return mx8


def apb_mx8_dequantize(mx8: torch.Tensor, rows: int, K: int, dtype: torch.dtype = torch.float32,
                       X: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    X, ptr, t, ld = _result(X, (rows, K), dtype, mx8, "X", stream)
    _check(load().apb_mx8_dequantize(_mx8_ptr(mx8, rows, K, "mx8"), int(rows), int(K), t, ptr, ld, _stream_at(stream, mx8, X)),
           "apb_mx8_dequantize")
    return X


# ----------------------------------------------------------------------------- gated feed-forward blocks

# "gelu" is the form by the hyperbolic tangent (torch.nn.GELU(approximate="tanh")), not the one by the error function.
_ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}                      # apb_activation


def _activation(name: str) -> int:
    a = _ACTIVATIONS.get(name)
    if a is None:
        raise ValueError("activation must be 'silu', 'gelu' or 'relu'")
    return a


def apb_mx4_gated_gemm(A: torch.Tensor, W: torch.Tensor, M: int, N: int, K: int, activation: str = "silu",
                       dtype: torch.dtype = torch.float32, Y: Optional[torch.Tensor] = None,
                       offsets: Optional[torch.Tensor] = None, saved: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Y[M, N] = act(A^ Wg^T) * (A^ Wu^T); W: for every expert N rows of the gate, then N of the up projection.  activation: "silu", "gelu"
    (the tanh form, 0.5 x (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3)))) or "relu", here and in what follows.  saved: memory from
    alloc_mx8(2 * M, N) that receives both projections in 8 bits for apb_gated_backward."""
    off, E = _experts(offsets)
    act = _activation(activation)
    if int(K) >> 31:
        raise ApbError(APB_ERR_SHAPE, "apb_mx4_gated_gemm")
    Y, ptr, t, ld = _result(Y, (M, N), dtype, A, "Y", stream)
    _check(load().apb_mx4_gated_gemm(_mx4_ptr(A, M, K, "A"), _mx4_ptr(W, E * 2 * N, K, "W"), off, E, int(M), int(N), int(K), act, t, ptr,
                                     ld, _mx8_ptr(saved, 2 * M, N, "saved"), _stream_at(stream, A, W, offsets, Y, saved)), "apb_mx4_gated_gemm")
    return Y


def apb_mx4_gated_linear_scratch_bytes(grouped: bool, E: int, M: int, N: int, K: int, with_saved: bool = False) -> int:
    """Bytes of scratch that apb_mx4_gated_linear uses: 0 where it runs as one kernel, and for sizes that it refuses."""
    if (E | M | N | K) >> 31:
        return 0
    return int(load().apb_mx4_gated_linear_scratch_bytes(int(grouped), E, M, N, K, int(with_saved)))


def apb_mx4_gated_linear(X: torch.Tensor, W: torch.Tensor, N: int, activation: str = "silu", dtype: Optional[torch.dtype] = None,
                         Y: Optional[torch.Tensor] = None, rows_from: Optional[torch.Tensor] = None,
                         offsets: Optional[torch.Tensor] = None, scratch: Optional[torch.Tensor] = None,
                         saved: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """apb_mx4_quantize of X [rows_in, K] + apb_mx4_gated_gemm with the 4-bit weights W in one call; Y has X's type by default."""
    xp, xt, ldx = _matrix(X, "X")
    rows_in, K = X.shape
    M = rows_in if rows_from is None else rows_from.numel()
    off, E = _experts(offsets)
    act = _activation(activation)
    lib, wp = load(), _mx4_ptr(W, E * 2 * N, K, "W")
    need = lib.apb_mx4_gated_linear_scratch_bytes(off is not None, E, M, N, K, saved is not None)
    if scratch is not None:
        sp = _array(scratch, torch.uint8, None, "scratch")
        if scratch.numel() < need:
            raise ValueError("scratch smaller than apb_mx4_gated_linear_scratch_bytes(...)")
    else:
        scratch = _new(X, need, torch.uint8, stream) if need else None
        sp = scratch.data_ptr() if need else wp                       # (none needed: not touched, but not NULL)
    Y, yp, yt, ldy = _result(Y, (M, N), dtype or X.dtype, X, "Y", stream)
    _check(lib.apb_mx4_gated_linear(xp, xt, ldx, rows_in, _array(rows_from, torch.int32, M, "rows_from"), wp, off, E, M, int(N), K, act,
                                    sp if need else wp, yt, yp, ldy, _mx8_ptr(saved, 2 * M, N, "saved"),
                                    _stream_at(stream, X, W, rows_from, offsets, scratch, Y, saved)), "apb_mx4_gated_linear")
    return Y


def apb_gated_forward(GU: torch.Tensor, activation: str = "silu", Y: Optional[torch.Tensor] = None,
                      saved: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Y[M, N] = act(G) * U from [G | U] = GU [M, 2N], in GU's type.  saved: as in apb_mx4_gated_gemm."""
    gp, gt, ldg = _matrix(GU, "GU")
    M, N = GU.shape[0], GU.shape[1] // 2
    if GU.shape[1] % 2:
        raise ValueError("GU must have an even number of columns")
    act = _activation(activation)
    Y, yp, yt, ldy = _result(Y, (M, N), GU.dtype, GU, "Y", stream)
    if yt != gt:
        raise TypeError("Y must have GU's type")
    _check(load().apb_gated_forward(gp, gt, ldg, M, N, act, yp, ldy, _mx8_ptr(saved, 2 * M, N, "saved"), _stream_at(stream, GU, Y, saved)),
           "apb_gated_forward")
    return Y


def apb_gated_backward(GU: torch.Tensor, dY: torch.Tensor, activation: str = "silu", dGU: Optional[torch.Tensor] = None,
                       Y: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """dGU [M, 2N] = [dG | dU] in dY's type, from dY [M, N] and GU: what `saved` has received (uint8), or a matrix [G | U].
    Y: if given, receives act(G) * U over again."""
    dp, dt, ldd = _matrix(dY, "dY")
    M, N = dY.shape
    act = _activation(activation)
    if GU.dtype == torch.uint8:
        gp, gt, ldg = _mx8_ptr(GU, 2 * M, N, "GU"), _MX8, 2 * N
    else:
        gp, gt, ldg = _matrix(GU, "GU")
        if tuple(GU.shape) != (M, 2 * N):
            raise ValueError("GU must be [M, 2N]")
    dGU, op, ot, ldo = _result(dGU, (M, 2 * N), dY.dtype, dY, "dGU", stream)
    yp, yt, ldy = None, dt, N
    if Y is not None:
        Y, yp, yt, ldy = _result(Y, (M, N), dY.dtype, dY, "Y", stream)
    if ot != dt or yt != dt:
        raise TypeError("dGU and Y must have dY's type")
    _check(load().apb_gated_backward(gp, gt, ldg, dp, dt, ldd, M, N, act, op, ldo, yp, ldy, _stream_at(stream, GU, dY, dGU, Y)), "apb_gated_backward")
    return dGU


# ----------------------------------------------------------------------------- low-rank adapters

def _factors(F: torch.Tensor, type_: torch.dtype, name: str) -> Tuple[int, int, int, int]:
    """(pointer, L, r, long side) of an adapters' factor."""
    if F.dim() != 3:
        raise ValueError(f"{name} must be [L, r, long side]")
    L, r, side = F.shape
    if (L | r | side) >> 31:
        raise ApbError(APB_ERR_SHAPE, name)
    return _array(F, type_, None, name), L, r, side


def _segments(offsets: Optional[torch.Tensor], adapter: Optional[torch.Tensor]):
    """(pointer of offsets, pointer of adapter, number of segments)."""
    if offsets is None:
        return None, _array(adapter, torch.int32, 1, "adapter"), 1
    S = offsets.numel() - 1
    if S < 1:
        raise ValueError("offsets must hold S + 1 int32")
    if S >> 31:
        raise ApbError(APB_ERR_SHAPE, "offsets")
    return _array(offsets, torch.int32, None, "offsets"), _array(adapter, torch.int32, S, "adapter"), S


def _low_rank(T: torch.Tensor) -> Tuple[int, int, int, int]:
    """(pointer, parts, M, r) of what apb_adapter_down returned."""
    if T.dim() != 3:
        raise ValueError("T must be [parts, M, r]")
    parts, M, r = T.shape
    if (parts | M | r) >> 31:
        raise ApbError(APB_ERR_SHAPE, "T")
    return _array(T, torch.float32, None, "T"), parts, M, r


def apb_adapter_parts(S: int, M: int, K: int, r: int) -> int:
    sizes = int(S), int(M), int(K), int(r)
    return 0 if any(n >> 31 for n in sizes) else int(load().apb_adapter_parts(*sizes))


def apb_adapter_down(X: torch.Tensor, A: torch.Tensor, offsets: Optional[torch.Tensor] = None, adapter: Optional[torch.Tensor] = None,
                     scale: Optional[torch.Tensor] = None, T: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """T = scale[a] X A[a]^T for X [M, K] and A [L, r, K], a the adapter of the row's segment (offsets int32 [S+1], adapter int32 [S]):
    float32 [parts, M, r], whose sum over the parts it is."""
    xp, xt, ldx = _matrix(X, "X")
    M, K = X.shape
    ap, L, r, k = _factors(A, X.dtype, "A")
    if k != K:
        raise ValueError("A must be [L, r, K]")
    off, adp, S = _segments(offsets, adapter)
    lib = load()
    parts = lib.apb_adapter_parts(S, M, K, r)
    if T is None:
        if parts == 0:
            raise ApbError(APB_ERR_SHAPE, "apb_adapter_down")
        T = _new(X, (parts, M, r), torch.float32, stream)
        tp = T.data_ptr()
    elif T.shape != (parts, M, r):
        raise ValueError(f"T must be [{parts}, {M}, {r}]")
    else:
        tp = _array(T, torch.float32, None, "T")
    _check(lib.apb_adapter_down(xp, xt, ldx, ap, off, adp, _array(scale, torch.float32, L, "scale"), S, L, M, K, r, tp,
                                _stream_at(stream, X, A, offsets, adapter, scale, T)), "apb_adapter_down")
    return T


def apb_adapter_up(T: torch.Tensor, B: torch.Tensor, Y0: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None,
                   offsets: Optional[torch.Tensor] = None, adapter: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Y = Y0 + T B[a] for B [L, r, N], in B's type (Y0 None: zeros).  Y may be Y0: rows without an adapter are then not touched."""
    tp, parts, M, r = _low_rank(T)
    bp, L, rb, N = _factors(B, B.dtype, "B")
    if rb != r:
        raise ValueError("B must be [L, r, N]")
    off, adp, S = _segments(offsets, adapter)
    p0, ld0 = None, N
    if Y0 is not None:
        if Y0.shape != (M, N) or Y0.dtype != B.dtype:
            raise ValueError("Y0 must be [M, N] in B's type")
        p0, _, ld0 = _matrix(Y0, "Y0")
    Y, yp, yt, ldy = _result(Y, (M, N), B.dtype, B, "Y", stream)
    if Y.dtype != B.dtype:
        raise TypeError("Y must have B's type")
    _check(load().apb_adapter_up(tp, parts, bp, yt, off, adp, S, L, M, N, r, p0, ld0, yp, ldy,
                                 _stream_at(stream, T, B, Y0, Y, offsets, adapter)), "apb_adapter_up")
    return Y


def apb_adapter_gradient_workspace_bytes(S: int, L: int, M: int, K: int, r: int) -> int:
    """Bytes of scratch that apb_adapter_gradient has a use for."""
    sizes = int(S), int(L), int(M), int(K), int(r)
    return 0 if any(n >> 31 for n in sizes) else int(load().apb_adapter_gradient_workspace_bytes(*sizes))


def apb_adapter_gradient(T: torch.Tensor, X: torch.Tensor, L: int, K: Optional[int] = None, offsets: Optional[torch.Tensor] = None,
                         adapter: Optional[torch.Tensor] = None, dA: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """dA[a] = sum over a's rows of T^T X, float32 [L, r, K].  X: [M, K], or its 8-bit form (uint8) with K given."""
    tp, parts, M, r = _low_rank(T)
    if X.dtype == torch.uint8:
        if K is None:
            raise ValueError("K must be given for an 8-bit X")
        xp, xt, ldx = _mx8_ptr(X, M, K, "X"), _MX8, K
    else:
        xp, xt, ldx = _matrix(X, "X")
        if X.shape[0] != M or K not in (None, X.shape[1]):
            raise ValueError("X must be [M, K]")
        K = X.shape[1]
    off, adp, S = _segments(offsets, adapter)
    lib = load()
    if L <= 0 or (int(L) | int(K)) >> 31:
        raise ApbError(APB_ERR_SHAPE, "apb_adapter_gradient")
    if dA is None:
        dA = _new(T, (L, r, K), torch.float32, stream)
        dp = dA.data_ptr()
    elif dA.shape != (L, r, K):
        raise ValueError(f"dA must be [{L}, {r}, {K}]")
    else:
        dp = _array(dA, torch.float32, None, "dA")
    keep, sp, sb = _scratch(workspace, lib.apb_adapter_gradient_workspace_bytes(S, L, M, K, r), T, stream)
    _check(lib.apb_adapter_gradient(tp, parts, xp, xt, ldx, off, adp, S, int(L), M, int(K), r, dp, sp, sb,
                                    _stream_at(stream, T, X, offsets, adapter, dA, keep)), "apb_adapter_gradient")
    return dA

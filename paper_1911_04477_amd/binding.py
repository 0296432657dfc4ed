"""Thin ctypes binding of libbnn.so: argument marshalling only.

Every function takes torch tensors that already live on the GPU, passes their
data pointers, sizes and the current HIP stream to the C entry point of the same
name, and raises ``BnnError`` on a non-zero status.  No arithmetic of the method
happens in Python, and there is no CPU fallback: if the HIP library has not been
built, loading fails loudly.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import warnings
from typing import List, Optional, Tuple

import torch

from .build import tensorcall_built_for

HERE = os.path.dirname(os.path.abspath(__file__))
# BNN_SANITIZE=1 (host-only checks, see build.py): the build whose host code carries ASan / UBSan
LIB_PATH = os.path.join(HERE, "libbnn_san.so" if os.environ.get("BNN_SANITIZE") == "1" else "libbnn.so")

_i64, _i32, _p, _sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t


class ChainLayer(ctypes.Structure):
    """bnn_chain_layer"""
    _fields_ = [("w_chain", _p), ("scale", _p), ("bias", _p), ("D", _i32), ("pool", _i32)]


class NormGateIn(ctypes.Structure):
    """bnn_norm_gate_in"""
    _fields_ = [("rows", _i64), ("D", _i32), ("type", _i32), ("r_type", _i32), ("post", _i32), ("pre", _i32),
                ("eps", ctypes.c_float), ("b", _p), ("b_ld", _i64), ("r", _p), ("r_ld", _i64), ("gate", _p), ("gate_ld", _i64),
                ("gate_rows", _i64), ("res_scale", _p), ("w_post", _p), ("bias_post", _p), ("w_pre", _p), ("bias_pre", _p)]


class F8Weight(ctypes.Structure):
    """bnn_f8_weight"""
    _fields_ = [("q", _p), ("ld", _i64), ("expert_ld", _i64), ("scale", _p), ("scale_ld", _i64), ("scale_expert_ld", _i64)]


# name -> (restype, argtypes); the list mirrors include/bnn.h one to one.
SIGNATURES = {
    "bnn_status_str": (ctypes.c_char_p, [_i32]),
    "bnn_packed_words": (_i64, [_i64]),
    "bnn_conv_kwords": (_i64, [_i32, _i32, _i32]),
    "bnn_conv_out_dim": (_i64, [_i64, _i64, _i64, _i64]),
    "bnn_encode": (_i32, [_p, _i64, _i64, _i64, _p, _i64, _p]),
    "bnn_pack_conv_weight": (_i32, [_p, _i32, _i32, _i32, _i32, _p, _p]),
    "bnn_im2col_packed": (_i32, [_p] + [_i32] * 10 + [_p, _p, _sz, _p]),
    "bnn_im2col_workspace_bytes": (_sz, [_i32] * 10),
    "bnn_xnor_gemm": (_i32, [_p, _i64, _p, _i64, _p, _i64, _i64, _i64, _i64, _p]),
    "bnn_xnor_gemm_mfma_i8": (_i32, [_p, _i64, _p, _i64, _p, _i64, _i64, _i64, _i64, _p]),
    "bnn_xnor_gemm_mfma_fp4": (_i32, [_p, _i64, _p, _i64, _p, _i64, _i64, _i64, _i64, _p]),
    "bnn_fp4_row_bytes": (_i64, [_i64]),
    "bnn_expand_fp4": (_i32, [_p, _i64, _i64, _i64, _p, _i64, _p]),
    "bnn_xnor_gemm_mfma_fp4_expanded": (_i32, [_p, _i64, _p, _i64, _p, _i64, _i64, _i64, _i64, _p]),
    "bnn_conv2d_mfma_fp4_expanded": (_i32, [_p, _p] + [_i32] * 11 + [_p, _p]),
    "bnn_control_conv2d_f32": (_i32, [_p, _p] + [_i32] * 11 + [_p, _p]),
    "bnn_xnor_gemm_epilogue": (_i32, [_p, _i64, _p, _i64, _i64, _i64, _i64, _p, _i64, _p, _i64, _p, _p, _i32, _p]),
    "bnn_conv2d": (_i32, [_p, _p] + [_i32] * 11 + [_p, _p, _p, _p, _p, _sz, _p]),
    "bnn_conv2d_workspace_bytes": (_sz, [_i32] * 10),
    "bnn_conv2d_noalloc": (_i32, [_p, _p] + [_i32] * 11 + [_p, _p, _p, _p, _p]),
    "bnn_conv2d_noalloc_max_bytes": (_sz, []),
    "bnn_conv2d_packed": (_i32, [_p, _p] + [_i32] * 12 + [_p, _p, _p, _p, _p, _p]),
    "bnn_conv_chain_weight_bytes": (_sz, [_i32, _i32]),
    "bnn_pack_conv_chain_weight": (_i32, [_p, _i32, _i32, _p, _p]),
    "bnn_conv_chain_pays": (_i32, [_i32] * 5 + [ctypes.POINTER(ChainLayer)]),
    "bnn_conv_chain": (_i32, [_p] + [_i32] * 5 + [ctypes.POINTER(ChainLayer), _p, _p]),
    "bnn_conv2d_f32_sign": (_i32, [_p, _p] + [_i32] * 11 + [_p, _p, _p, _p]),
    "bnn_pack_fc_weight_nhwc": (_i32, [_p, _i64, _i32, _i32, _i32, _p, _p]),
    "bnn_maxpool2x2": (_i32, [_p, _i32, _i32, _i32, _i32, _p, _p, _p, _p, _p]),
    "bnn_conv2d_f32": (_i32, [_p, _p] + [_i32] * 11 + [_p, _p, _p, _p]),
    "bnn_fc_f32": (_i32, [_p, _p, _p, _i64, _i64, _i64, _i32, _p, _p]),
    "bnn_quant_rows_i8": (_i32, [_p, _i32, _i64, _i64, _i64, _p, _i64, _p, _p]),
    "bnn_linear_i8": (_i32, [_p, _i64, _p, _p, _i64, _p, _p, _i64, _i64, _i64, _p, _i32, _i64, _p]),
    "bnn_norm_gate": (_i32, [ctypes.POINTER(NormGateIn), _p, _i64, _p, _i64, _p, _i64, _p, _p]),
    "bnn_norm_gate_backward": (_i32, [ctypes.POINTER(NormGateIn), _p, _i64, _p, _i64, _p, _i64, _p, _i64, _p, _i64, _p, _p,
                                      _p, _p, _p, _p, _sz, _p]),
    "bnn_norm_gate_backward_workspace_bytes": (_sz, [_i64, _i32, _i64]),
    "bnn_gated_ff_saved_bytes": (_sz, [_i64, _i64]),
    "bnn_gated_ff": (_i32, [_p, _i64, _p, _i64, _p, _i64, _i32, _i64, _i64, _i64, _i32, _p, _i64, _p, _p]),
    "bnn_gated_ff_i8": (_i32, [_p, _i64, _p, _p, _i64, _p, _p, _i64, _p, _i64, _i64, _i64, _i32, _p, _i32, _i64, _p]),
    "bnn_gated_ff_backward_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "bnn_gated_ff_backward": (_i32, [_p, _i64, _p, _i64, _p, _i64, _i32, _i64, _i64, _i64, _p, _p, _i64, _p, _i64, _p, _i64,
                                     _p, _i64, _p, _sz, _p]),
    "bnn_f8_row_bytes": (_i64, [_i64]),
    "bnn_f8_scale_bytes": (_i64, [_i64]),
    "bnn_quant_blocks_f8": (_i32, [_p, _i32, _i64, _i64, _p, _i64, _i64, _i64, _p, _i64, _p, _i64, _p]),
    "bnn_quant_columns_f8": (_i32, [_p, _i32, _i64, _i64, _p, _i64, _i64, _i64, _p, _i64, _p, _i64, _p]),
    "bnn_quant_weight_f8": (_i32, [_p, _i32, _i64, _i64, _i64, _i64, _i64, ctypes.POINTER(F8Weight), ctypes.POINTER(F8Weight), _p]),
    "bnn_linear_f8": (_i32, [_p, _i64, _p, _i64, _p, _i64, _p, _i32, _i64, _i32, _p, _i64, _i64, _i64, _p, _i32, _i64, _p]),
    "bnn_expert_linear_f8": (_i32, [_p, _i64, _p, _i64, _p, _i64, _p, _i64, _i64, _p, _i32, _i64, _i64, _i32, _i64, _i64, _i64, _p,
                                    _i32, _i64, _p]),
    "bnn_expert_linear_f8_dw": (_i32, [_p, _i64, _p, _i64, _p, _i64, _p, _i64, _p, _i64, _i64, _i64, _i64, _p, _i32, _i64, _i64, _p]),
    "bnn_expert_rows": (_i64, [_i64, _i64, _i64, _i64]),
    "bnn_expert_sort_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "bnn_expert_sort": (_i32, [_p, _i32, _i64, _i64, _i64, _i64, _i64, _p, _p, _p, _p, _sz, _p]),
    "bnn_expert_gather": (_i32, [_p, _i32, _i64, _i64, _p, _i64, _i64, _i64, _p, _i64, _p]),
    "bnn_expert_combine": (_i32, [_p, _i32, _i64, _i64, _p, _p, _i64, _i64, _i64, _p, _i64, _p]),
    "bnn_expert_combine_backward": (_i32, [_p, _i32, _i64, _i64, _p, _p, _p, _p, _i64, _i64, _i64, _i64, _p, _i64, _p, _p]),
    "bnn_gated_act": (_i32, [_p, _i32, _i64, _i64, _i64, _i32, _p, _p, _i64, _p]),
    "bnn_gated_act_f8": (_i32, [_p, _i32, _i64, _i64, _i64, _i32, _p, _p, _i64, _p, _i64, _p]),
    "bnn_gated_act_backward": (_i32, [_p, _i32, _i64, _i64, _i64, _i32, _p, _p, _i64, _p, _i64, _p]),
}

# include/bnn_testing.h: the same calls with the kernel variant chosen by the caller, the
# kernel-timing hook and the two yardstick kernels.  Tests and bench.py only.
TESTING_SIGNATURES = {
    "bnn_testing_xnor_gemm_epilogue": (_i32, [_p, _i64, _p, _i64, _i64, _i64, _i64, _p, _i64, _p, _i64, _p, _p, _i32,
                                              _i32, _p]),
    "bnn_testing_conv2d": (_i32, [_p, _p] + [_i32] * 11 + [_p, _p, _p, _p, _p, _sz, _i32, _i32, _p]),
    "bnn_testing_conv2d_packed": (_i32, [_p, _p] + [_i32] * 12 + [_p, _p, _p, _p, _p, _i32, _i32, _p]),
    "bnn_testing_conv_image": (_i32, [_i32] * 14 + [ctypes.POINTER(_i64)]),
    "bnn_testing_conv_word": (_i32, [_i32] * 14),
    "bnn_testing_conv_word_nontemporal": (_i32, [_i32] * 11),
    "bnn_testing_first_sign": (_i32, [_i32] * 9),
    "bnn_testing_conv_region": (_i32, [_i32] * 12 + [ctypes.POINTER(_i64)]),
    "bnn_testing_nontemporal_maps": (_i32, [_i32, _i32, _i32, _i64, _i64]),
    "bnn_testing_xnor_gemm_mfma_fp4_expanded": (_i32, [_p, _i64, _p, _i64, _p, _i64, _i64, _i64, _i64, _i32, _p]),
    "bnn_testing_product_form": (_i32, [_i64, _i64, _i32, _i32, _i32]),
    "bnn_testing_gated_backward_plan": (_i32, [_i64, _i64, _i64, ctypes.POINTER(_i64)]),
    "bnn_testing_f8_form": (_i32, [_i64, _i64, _i32, _i64, _i64, _i32, _i32, _i32]),
    "bnn_prof_enable": (_i32, [_i32]),
    "bnn_prof_reset": (_i32, []),
    "bnn_prof_count": (_i64, []),
    "bnn_prof_get": (_i32, [_i64, ctypes.POINTER(_i32), ctypes.POINTER(ctypes.c_float)]),
    "bnn_kernel_name": (ctypes.c_char_p, [_i32]),
    "bnn_valu_peak_probe": (_i32, [_p, _i32, _i32, _i32, _p]),
    "bnn_copy_probe": (_i32, [_p, _p, _sz, _p]),
}

BNN_OK = 0
CH_NONE, CH_ROW, CH_COL = 0, 1, 2

_lib: Optional[ctypes.CDLL] = None


FASTCALL_PATH = LIB_PATH.replace("libbnn", "_fastcall")
TENSORCALL_PATH = LIB_PATH.replace("libbnn", "_tensorcall")


def _fastcall():
    """The call helper, or None (with a warning) where only libbnn has been built."""
    if not os.path.exists(FASTCALL_PATH):
        warnings.warn(f"{FASTCALL_PATH} is missing: build it with `python paper_1911_04477_amd/build.py`; until then calls "
                      "go through ctypes, 0.4 to 0.9 us slower each", RuntimeWarning, stacklevel=4)
        return None
    spec = importlib.util.spec_from_file_location("paper_1911_04477_amd._fastcall", FASTCALL_PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


class _Calls:
    """The functions of SIGNATURES and TESTING_SIGNATURES whose arguments are integers and raw pointers, called without
    ctypes' conversions (csrc/fastcall.c)."""

    _KINDS = {_p: "p", _i64: "q", _i32: "i", _sz: "z"}

    def __init__(self, L: ctypes.CDLL):
        fast = _fastcall()
        for name, (res, args) in list(SIGNATURES.items()) + list(TESTING_SIGNATURES.items()):
            args = [_p if isinstance(a, type) and issubclass(a, ctypes._Pointer) else a for a in args]
            if res not in (_i32, _i64, _sz) or any(a not in self._KINDS for a in args):
                continue
            address = ctypes.cast(getattr(L, name), ctypes.c_void_p).value
            setattr(self, name, fast.Function(address, "".join(self._KINDS[a] for a in args), "i" if res is _i32 else "q")
                    if fast else ctypes.CFUNCTYPE(res, *args)(address))


_calls: Optional[_Calls] = None


def _c() -> _Calls:
    global _calls
    if _calls is None:
        _calls = _Calls(lib())
    return _calls


class _Tensors:
    """Calls from the tensors themselves (csrc/tensorcall.cpp): a status (the gradients: their tensors, or a status), or None where
    the call is not a plain one and the function of this module has to look at it.  Where the extension has not been built, or for
    another torch, every call is of that kind."""

    FUNCTIONS = ("gemm", "epilogue", "encode", "conv2d", "conv2d_packed", "im2col", "f32_sign", "conv2d_f32", "maxpool", "fc",
                 "quant_rows", "linear_i8", "norm_gate", "norm_gate_backward", "norm_gate_gradients", "gated_ff", "gated_ff_i8",
                 "gated_ff_backward", "gated_ff_gradients", "quant_f8", "linear_f8", "expert_linear_f8", "expert_linear_f8_dw", "expert_sort",
                 "expert_gather", "expert_combine", "expert_combine_backward", "gated_act", "gated_act_f8", "gated_act_backward")

    def __init__(self, L: ctypes.CDLL, path: str):
        module = None
        if os.path.exists(path):
            try:
                spec = importlib.util.spec_from_file_location("paper_1911_04477_amd._tensorcall", path)
                module = importlib.util.module_from_spec(spec)
                spec.loader.exec_module(module)
                if module.built_for != tensorcall_built_for(torch):  # it would read tensors at wrong places
                    raise ImportError(f"built for {module.built_for}")
            except (ImportError, AttributeError) as e:  # of another torch or Python
                module = None
                warnings.warn(f"{path} does not load ({e}): build it again; calls take 1 to 2 us longer", RuntimeWarning, stacklevel=4)
        if module is not None:
            module.bind(*[ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in module.names])
        for f in self.FUNCTIONS:
            setattr(self, f, getattr(module, f) if module is not None else lambda *args: None)


_tensors: Optional[_Tensors] = None


def _t() -> _Tensors:
    global _tensors
    if _tensors is None:
        _tensors = _Tensors(lib(), TENSORCALL_PATH)
    return _tensors


class BnnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        name = lib().bnn_status_str(self.status).decode()
        super().__init__(f"{where} failed: {name} ({self.status})")


def lib() -> ctypes.CDLL:
    """Load libbnn.so (built by paper_1911_04477_amd/build.py).  No fallback."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python paper_1911_04477_amd/build.py` "
                "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in list(SIGNATURES.items()) + list(TESTING_SIGNATURES.items()):
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(st: int, where: str) -> None:
    if st != BNN_OK:
        raise BnnError(st, where)


def _stream() -> int:
    # the current stream of the current device as a raw handle: torch.cuda.current_stream() builds a Stream object
    # on every call, 2.7 of the 8.4 us that a whole call through this binding took (0.1 us this way)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dev(t: torch.Tensor, dtype: torch.dtype, name: str) -> None:
    if not t.is_cuda or t.dtype != dtype:
        raise TypeError(f"{name} must be a GPU tensor of dtype {dtype}")


def packed_words(K: int) -> int:
    return _c().bnn_packed_words(K)


def conv_kwords(C: int, kH: int, kW: int) -> int:
    return int(_c().bnn_conv_kwords(C, kH, kW))


def conv_out_dim(n: int, k: int, s: int, p: int) -> int:
    return int(_c().bnn_conv_out_dim(n, k, s, p))


def bnn_encode(src: torch.Tensor, dst: Optional[torch.Tensor] = None) -> torch.Tensor:
    """src fp32 [rows, K] (row stride = src.stride(0)) -> int64-typed packed words [rows, Kw]."""
    if dst is not None:
        st = _t().encode(src, dst)
        if st is not None:
            _check(st, "bnn_encode")
            return dst
    _dev(src, torch.float32, "src")
    assert src.dim() == 2 and src.stride(1) == 1
    rows, K = src.shape
    Kw = packed_words(K)
    if dst is None:
        dst = torch.empty((rows, Kw), dtype=torch.int64, device=src.device)
    _dev(dst, torch.int64, "dst")
    assert dst.stride(1) == 1
    _check(_c().bnn_encode(_ptr(src), rows, K, src.stride(0) if rows > 1 else max(K, src.stride(0)), _ptr(dst),
                            dst.stride(0) if rows > 1 else max(Kw, dst.stride(0)), _stream()), "bnn_encode")
    return dst


def bnn_pack_conv_weight(w: torch.Tensor) -> torch.Tensor:
    _dev(w, torch.float32, "w")
    assert w.dim() == 4 and w.is_contiguous()
    D, C, kH, kW = w.shape
    out = torch.empty((D, conv_kwords(C, kH, kW)), dtype=torch.int64, device=w.device)
    _check(_c().bnn_pack_conv_weight(_ptr(w), D, C, kH, kW, _ptr(out), _stream()), "bnn_pack_conv_weight")
    return out


def im2col_workspace_bytes(x_shape, kH, kW, stride, pad) -> int:
    N, C, H, W = x_shape
    return int(_c().bnn_im2col_workspace_bytes(N, C, H, W, kH, kW, stride[0], stride[1], pad[0], pad[1]))


def bnn_im2col_packed(x: torch.Tensor, kH: int, kW: int, stride=(1, 1), pad=(0, 0),
                      cols: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    if cols is not None and workspace is not None:
        st = _t().im2col(x, kH, kW, stride, pad, cols, workspace)
        if st is not None:
            _check(st, "bnn_im2col_packed")
            return cols
    _dev(x, torch.float32, "x")
    assert x.dim() == 4 and x.is_contiguous()
    N, C, H, W = x.shape
    geo = (N, C, H, W, kH, kW, stride[0], stride[1], pad[0], pad[1])
    OH, OW = conv_out_dim(H, kH, stride[0], pad[0]), conv_out_dim(W, kW, stride[1], pad[1])
    if cols is None:
        cols = torch.empty((N * OH * OW, conv_kwords(C, kH, kW)), dtype=torch.int64, device=x.device)
    _dev(cols, torch.int64, "cols")
    assert cols.is_contiguous() and cols.numel() == N * OH * OW * conv_kwords(C, kH, kW)
    nbytes = int(_c().bnn_im2col_workspace_bytes(*geo))
    if workspace is None:
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=x.device)
    _check(_c().bnn_im2col_packed(_ptr(x), *geo, _ptr(cols), _ptr(workspace), workspace.numel(), _stream()),
           "bnn_im2col_packed")
    return cols


def bnn_xnor_gemm(A: torch.Tensor, B: torch.Tensor, K: int, C: Optional[torch.Tensor] = None,
                  cfg: Optional[int] = None) -> torch.Tensor:
    """A [M, >=Kw], B [N, >=Kw] packed (int64-typed) -> int32 [M, N].
    cfg (tests only): the same call through bnn_testing_xnor_gemm_epilogue on that tile configuration."""
    if C is not None and cfg is None:
        st = _t().gemm(A, B, K, C)
        if st is not None:
            _check(st, "bnn_xnor_gemm")
            return C
    _dev(A, torch.int64, "A")
    _dev(B, torch.int64, "B")
    M, N = A.shape[0], B.shape[0]
    if C is None:
        C = torch.empty((M, N), dtype=torch.int32, device=A.device)
    _dev(C, torch.int32, "C")
    lda = A.stride(0) if M > 1 else max(A.shape[1], 1)
    ldb = B.stride(0) if N > 1 else max(B.shape[1], 1)
    ldc = C.stride(0) if M > 1 else max(N, 1)
    if cfg is None:
        _check(_c().bnn_xnor_gemm(_ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, M, N, K, _stream()), "bnn_xnor_gemm")
    else:
        _check(_c().bnn_testing_xnor_gemm_epilogue(_ptr(A), lda, _ptr(B), ldb, M, N, K, _ptr(C), ldc, None, 0, None,
                                                    None, CH_NONE, cfg, _stream()), "bnn_testing_xnor_gemm_epilogue")
    return C


def bnn_xnor_gemm_mfma_i8(A: torch.Tensor, B: torch.Tensor, K: int, C: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Ablation: same contract as bnn_xnor_gemm, computed with int8 MFMA."""
    _dev(A, torch.int64, "A")
    _dev(B, torch.int64, "B")
    M, N = A.shape[0], B.shape[0]
    if C is None:
        C = torch.empty((M, N), dtype=torch.int32, device=A.device)
    lda = A.stride(0) if M > 1 else max(A.shape[1], 1)
    ldb = B.stride(0) if N > 1 else max(B.shape[1], 1)
    _check(_c().bnn_xnor_gemm_mfma_i8(_ptr(A), lda, _ptr(B), ldb, _ptr(C), C.stride(0) if M > 1 else max(N, 1), M, N,
                                       K, _stream()), "bnn_xnor_gemm_mfma_i8")
    return C


def bnn_xnor_gemm_mfma_fp4(A: torch.Tensor, B: torch.Tensor, K: int, C: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Ablation: same contract as bnn_xnor_gemm, computed with the 4-bit floating-point MFMA."""
    _dev(A, torch.int64, "A")
    _dev(B, torch.int64, "B")
    M, N = A.shape[0], B.shape[0]
    if C is None:
        C = torch.empty((M, N), dtype=torch.int32, device=A.device)
    lda = A.stride(0) if M > 1 else max(A.shape[1], 1)
    ldb = B.stride(0) if N > 1 else max(B.shape[1], 1)
    _check(_c().bnn_xnor_gemm_mfma_fp4(_ptr(A), lda, _ptr(B), ldb, _ptr(C), C.stride(0) if M > 1 else max(N, 1), M, N,
                                        K, _stream()), "bnn_xnor_gemm_mfma_fp4")
    return C


def bnn_expand_fp4(packed: torch.Tensor, K: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Ablation: packed sign rows [rows, >= ceil(K/64)] int64 -> E2M1 rows [rows, 32 * ceil(K/64)] uint8."""
    _dev(packed, torch.int64, "packed")
    rows = packed.shape[0]
    rb = int(_c().bnn_fp4_row_bytes(K))
    if out is None:
        out = torch.empty((rows, rb), dtype=torch.uint8, device=packed.device)
    src_ld = packed.stride(0) if rows > 1 else max(packed.shape[1], 1)
    dst_ld = out.stride(0) if rows > 1 else max(out.shape[1], 16)
    _check(_c().bnn_expand_fp4(_ptr(packed), rows, K, src_ld, _ptr(out), dst_ld, _stream()), "bnn_expand_fp4")
    return out


def bnn_xnor_gemm_mfma_fp4_expanded(A4: torch.Tensor, B4: torch.Tensor, K: int, C: Optional[torch.Tensor] = None,
                                    tile: Optional[int] = None) -> torch.Tensor:
    """Ablation: the binarized GEMM on operands kept in memory as E2M1 +-1 rows (bnn_expand_fp4)."""
    _dev(A4, torch.uint8, "A4")
    _dev(B4, torch.uint8, "B4")
    M, N = A4.shape[0], B4.shape[0]
    if C is None:
        C = torch.empty((M, N), dtype=torch.int32, device=A4.device)
    lda = A4.stride(0) if M > 1 else max(A4.shape[1], 16)
    ldb = B4.stride(0) if N > 1 else max(B4.shape[1], 16)
    ldc = C.stride(0) if M > 1 else max(N, 1)
    if tile is None:
        _check(_c().bnn_xnor_gemm_mfma_fp4_expanded(_ptr(A4), lda, _ptr(B4), ldb, _ptr(C), ldc, M, N, K, _stream()),
               "bnn_xnor_gemm_mfma_fp4_expanded")
    else:
        _check(_c().bnn_testing_xnor_gemm_mfma_fp4_expanded(_ptr(A4), lda, _ptr(B4), ldb, _ptr(C), ldc, M, N, K, tile,
                                                             _stream()), "bnn_testing_xnor_gemm_mfma_fp4_expanded")
    return C


def bnn_conv2d_mfma_fp4_expanded(x4: torch.Tensor, w4: torch.Tensor, C: int, D: int, kH: int, kW: int, stride=(1, 1),
                                 pad=(0, 0), out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Ablation: x4 [N, H, W, C/2] uint8 (E2M1 codes), w4 [D, kH*kW*C/2] uint8 -> int32 NCHW."""
    _dev(x4, torch.uint8, "x4")
    _dev(w4, torch.uint8, "w4")
    assert x4.dim() == 4 and x4.is_contiguous() and w4.is_contiguous()
    N, H, W, _ = x4.shape
    OH, OW = conv_out_dim(H, kH, stride[0], pad[0]), conv_out_dim(W, kW, stride[1], pad[1])
    if out is None:
        out = torch.empty((N, D, OH, OW), dtype=torch.int32, device=x4.device)
    _check(_c().bnn_conv2d_mfma_fp4_expanded(_ptr(x4), _ptr(w4), N, C, H, W, D, kH, kW, stride[0], stride[1], pad[0],
                                              pad[1], _ptr(out), _stream()), "bnn_conv2d_mfma_fp4_expanded")
    return out


def bnn_control_conv2d_f32(x: torch.Tensor, w: torch.Tensor, stride=(1, 1), pad=(0, 0),
                           out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Control group: the binarized convolution as an fp32 GEMM on sign(x), sign(w)."""
    _dev(x, torch.float32, "x")
    _dev(w, torch.float32, "w")
    N, C, H, W = x.shape
    D, _, kH, kW = w.shape
    OH, OW = conv_out_dim(H, kH, stride[0], pad[0]), conv_out_dim(W, kW, stride[1], pad[1])
    if out is None:
        out = torch.empty((N, D, OH, OW), dtype=torch.float32, device=x.device)
    _check(_c().bnn_control_conv2d_f32(_ptr(x), _ptr(w), N, C, H, W, D, kH, kW, stride[0], stride[1], pad[0], pad[1],
                                        _ptr(out), _stream()), "bnn_control_conv2d_f32")
    return out


def bnn_xnor_gemm_epilogue(A: torch.Tensor, B: torch.Tensor, K: int, scale: torch.Tensor, bias: torch.Tensor,
                           axis: int, want_int: bool = False, out_y: Optional[torch.Tensor] = None,
                           cfg: Optional[int] = None) -> Tuple[Optional[torch.Tensor], torch.Tensor]:
    if out_y is not None and not want_int and cfg is None:
        st = _t().epilogue(A, B, K, scale, bias, axis, out_y)
        if st is not None:
            _check(st, "bnn_xnor_gemm_epilogue")
            return None, out_y
    _dev(A, torch.int64, "A")
    _dev(B, torch.int64, "B")
    M, N = A.shape[0], B.shape[0]
    if out_y is not None:
        _dev(out_y, torch.float32, "out_y")
        assert out_y.shape == (M, N) and out_y.is_contiguous()
    Y = out_y if out_y is not None else torch.empty((M, N), dtype=torch.float32, device=A.device)
    C = torch.empty((M, N), dtype=torch.int32, device=A.device) if want_int else None
    lda = A.stride(0) if M > 1 else max(A.shape[1], 1)
    ldb = B.stride(0) if N > 1 else max(B.shape[1], 1)
    if cfg is None:
        _check(_c().bnn_xnor_gemm_epilogue(_ptr(A), lda, _ptr(B), ldb, M, N, K, _ptr(C), max(N, 1), _ptr(Y), max(N, 1),
                                            _ptr(scale), _ptr(bias), axis, _stream()), "bnn_xnor_gemm_epilogue")
    else:
        _check(_c().bnn_testing_xnor_gemm_epilogue(_ptr(A), lda, _ptr(B), ldb, M, N, K, _ptr(C), max(N, 1), _ptr(Y),
                                                    max(N, 1), _ptr(scale), _ptr(bias), axis, cfg, _stream()),
               "bnn_testing_xnor_gemm_epilogue")
    return C, Y


def conv2d_workspace_bytes(x_shape, kH, kW, stride, pad) -> int:
    N, C, H, W = x_shape
    return int(_c().bnn_conv2d_workspace_bytes(N, C, H, W, kH, kW, stride[0], stride[1], pad[0], pad[1]))


def bnn_conv2d(x: torch.Tensor, w_packed: torch.Tensor, D: int, kH: int, kW: int, stride=(1, 1), pad=(0, 0),
               scale: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, want_int: bool = True,
               workspace: Optional[torch.Tensor] = None, out_i32: Optional[torch.Tensor] = None,
               out_f32: Optional[torch.Tensor] = None, cfg: Optional[int] = None, lean: Optional[int] = None):
    """Returns (out_i32 or None, out_f32 or None), both NCHW.
    cfg / lean (tests only): the same call through bnn_testing_conv2d."""
    if (workspace is not None and (out_i32 is not None or not want_int) and (out_f32 is not None or scale is None)
            and cfg is None and lean is None):
        st = _t().conv2d(x, w_packed, D, kH, kW, stride, pad, out_i32, out_f32, scale, bias, workspace)
        if st is not None:
            _check(st, "bnn_conv2d")
            return out_i32, out_f32
    _dev(x, torch.float32, "x")
    _dev(w_packed, torch.int64, "w_packed")
    assert x.dim() == 4 and x.is_contiguous() and w_packed.is_contiguous()
    N, C, H, W = x.shape
    OH, OW = conv_out_dim(H, kH, stride[0], pad[0]), conv_out_dim(W, kW, stride[1], pad[1])
    nbytes = conv2d_workspace_bytes(x.shape, kH, kW, stride, pad)
    if workspace is None:
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=x.device)
    if want_int and out_i32 is None:
        out_i32 = torch.empty((N, D, OH, OW), dtype=torch.int32, device=x.device)
    if scale is not None and out_f32 is None:
        out_f32 = torch.empty((N, D, OH, OW), dtype=torch.float32, device=x.device)
    if cfg is None and lean is None:
        _check(_c().bnn_conv2d(_ptr(x), _ptr(w_packed), N, C, H, W, D, kH, kW, stride[0], stride[1], pad[0], pad[1],
                                _ptr(out_i32), _ptr(out_f32), _ptr(scale), _ptr(bias), _ptr(workspace),
                                workspace.numel(), _stream()), "bnn_conv2d")
    else:
        _check(_c().bnn_testing_conv2d(_ptr(x), _ptr(w_packed), N, C, H, W, D, kH, kW, stride[0], stride[1], pad[0],
                                        pad[1], _ptr(out_i32), _ptr(out_f32), _ptr(scale), _ptr(bias),
                                        _ptr(workspace), workspace.numel(), -1 if cfg is None else cfg,
                                        1 if lean is None else lean, _stream()), "bnn_testing_conv2d")
    return out_i32, out_f32


def bnn_conv2d_noalloc(x: torch.Tensor, w_packed: torch.Tensor, D: int, kH: int, kW: int, stride, pad,
                       out_i32: Optional[torch.Tensor], out_f32: Optional[torch.Tensor] = None,
                       scale: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None) -> None:
    """bnn_conv2d without a workspace argument; the caller passes every output buffer, so the call
    allocates nothing on either side of the ABI."""
    _dev(x, torch.float32, "x")
    _dev(w_packed, torch.int64, "w_packed")
    assert x.dim() == 4 and x.is_contiguous() and w_packed.is_contiguous()
    N, C, H, W = x.shape
    _check(_c().bnn_conv2d_noalloc(_ptr(x), _ptr(w_packed), N, C, H, W, D, kH, kW, stride[0], stride[1], pad[0],
                                    pad[1], _ptr(out_i32), _ptr(out_f32), _ptr(scale), _ptr(bias), _stream()),
           "bnn_conv2d_noalloc")


def bnn_conv2d_packed(xp: torch.Tensor, w_packed: torch.Tensor, C: int, D: int, kH: int, kW: int, stride=(1, 1),
                      pad=(0, 0), pool: int = 0, scale: Optional[torch.Tensor] = None,
                      bias: Optional[torch.Tensor] = None, out: str = "packed", out_buf: Optional[torch.Tensor] = None,
                      cfg: Optional[int] = None, lean: Optional[int] = None):
    """xp: packed NHWC [N, H, W, Cw] (int64-typed).  out = "packed" | "i32" | "f32".
    cfg / lean (tests only): the same call through bnn_testing_conv2d_packed."""
    if out_buf is not None and cfg is None and lean is None and out in ("packed", "i32", "f32"):
        st = _t().conv2d_packed(xp, w_packed, C, D, kH, kW, stride, pad, pool, out_buf if out == "i32" else None,
                                out_buf if out == "f32" else None, out_buf if out == "packed" else None, scale, bias)
        if st is not None:
            _check(st, "bnn_conv2d_packed")
            return out_buf
    _dev(xp, torch.int64, "x_packed")
    _dev(w_packed, torch.int64, "w_packed")
    assert xp.dim() == 4 and xp.is_contiguous() and w_packed.is_contiguous()
    N, H, W, Cw = xp.shape
    assert Cw == packed_words(C)
    OH, OW = conv_out_dim(H, kH, stride[0], pad[0]), conv_out_dim(W, kW, stride[1], pad[1])
    oi = of = op = None
    if out == "packed":
        op = out_buf if out_buf is not None else torch.empty(
            (N, OH // 2 if pool else OH, OW // 2 if pool else OW, packed_words(D)), dtype=torch.int64, device=xp.device)
    elif out == "i32":
        oi = out_buf if out_buf is not None else torch.empty((N, D, OH, OW), dtype=torch.int32, device=xp.device)
    elif out == "f32":
        of = out_buf if out_buf is not None else torch.empty((N, D, OH, OW), dtype=torch.float32, device=xp.device)
    else:
        raise ValueError(out)
    if cfg is None and lean is None:
        _check(_c().bnn_conv2d_packed(_ptr(xp), _ptr(w_packed), N, C, H, W, D, kH, kW, stride[0], stride[1], pad[0],
                                       pad[1], pool, _ptr(oi), _ptr(of), _ptr(op), _ptr(scale), _ptr(bias), _stream()),
               "bnn_conv2d_packed")
    else:
        _check(_c().bnn_testing_conv2d_packed(_ptr(xp), _ptr(w_packed), N, C, H, W, D, kH, kW, stride[0], stride[1],
                                               pad[0], pad[1], pool, _ptr(oi), _ptr(of), _ptr(op), _ptr(scale),
                                               _ptr(bias), -1 if cfg is None else cfg, 1 if lean is None else lean,
                                               _stream()), "bnn_testing_conv2d_packed")
    return op if op is not None else (oi if oi is not None else of)


def bnn_pack_conv_chain_weight(w_packed: torch.Tensor, C: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Filter bank of a 3x3 layer from bnn_pack_conv_weight, in the order in which bnn_conv_chain multiplies it."""
    _dev(w_packed, torch.int64, "w_packed")
    D = w_packed.shape[0]
    assert w_packed.is_contiguous() and w_packed.shape[1] == conv_kwords(C, 3, 3)
    if out is None:
        out = torch.empty(max(16, int(_c().bnn_conv_chain_weight_bytes(C, D))), dtype=torch.uint8, device=w_packed.device)
    else:
        _chain_weight(out, C, D)
    _check(_c().bnn_pack_conv_chain_weight(_ptr(w_packed), D, C, _ptr(out), _stream()), "bnn_pack_conv_chain_weight")
    return out


def _chain_weight(w: torch.Tensor, C: int, D: int) -> None:
    _dev(w, torch.uint8, "w_chain")
    need = int(_c().bnn_conv_chain_weight_bytes(C, D))
    if not w.is_contiguous() or w.numel() < need:
        raise ValueError(f"w_chain: {need} contiguous bytes for {C} to {D} channels")


def conv_chain_layers(layers) -> ctypes.Array:
    """[(w_chain or None, scale, bias, D, pool)] -> the host array bnn_conv_chain takes.  It holds the tensors whose
    addresses it contains (`tensors`), so they live as long as it does.  w_chain None: for bnn_conv_chain_pays alone."""
    layers = [tuple(L) for L in layers]
    for i, (w, s, b, D, pool) in enumerate(layers):
        for t, name in ((s, "scale"), (b, "bias")):
            _dev(t, torch.float32, name)
            if not t.is_contiguous() or t.numel() < D:
                raise ValueError(f"{name}: {D} contiguous values")
        if w is not None and i > 0:  # the first layer's: where its input channels are known
            _chain_weight(w, layers[i - 1][3], D)
    out = (ChainLayer * len(layers))(*[ChainLayer(_ptr(w), _ptr(s), _ptr(b), D, pool) for w, s, b, D, pool in layers])
    out.tensors = [L[:3] for L in layers]
    return out


def bnn_conv_chain_pays(N: int, C: int, H: int, W: int, layers: ctypes.Array) -> bool:
    return bool(_c().bnn_conv_chain_pays(N, C, H, W, len(layers), ctypes.addressof(layers)))


def bnn_conv_chain(xp: torch.Tensor, C: int, layers: ctypes.Array, out: torch.Tensor) -> torch.Tensor:
    """xp: packed NHWC [N, H, W, C / 64] through consecutive 3x3 layers; out: the last layer's packed map."""
    _dev(xp, torch.int64, "x_packed")
    _dev(out, torch.int64, "out")
    N, H, W, Cw = xp.shape
    assert xp.is_contiguous() and out.is_contiguous() and Cw == packed_words(C)
    held = getattr(layers, "tensors", None)  # an array of another origin is the caller's own
    if held and held[0][0] is not None:
        _chain_weight(held[0][0], C, layers[0].D)
    OH, OW = H, W
    for L in layers:
        if L.pool:
            OH, OW = OH // 2, OW // 2
    assert tuple(out.shape) == (N, OH, OW, packed_words(layers[-1].D))
    _check(_c().bnn_conv_chain(_ptr(xp), N, C, H, W, len(layers), ctypes.addressof(layers), _ptr(out), _stream()), "bnn_conv_chain")
    return out


def bnn_conv2d_f32_sign(x: torch.Tensor, w: torch.Tensor, scale: torch.Tensor, bias: torch.Tensor, stride=(1, 1),
                        pad=(0, 0), out: Optional[torch.Tensor] = None) -> torch.Tensor:
    if out is not None:
        st = _t().f32_sign(x, w, scale, bias, stride, pad, out)
        if st is not None:
            _check(st, "bnn_conv2d_f32_sign")
            return out
    _dev(x, torch.float32, "x")
    _dev(w, torch.float32, "w")
    N, C, H, W = x.shape
    D, _, kH, kW = w.shape
    OH, OW = conv_out_dim(H, kH, stride[0], pad[0]), conv_out_dim(W, kW, stride[1], pad[1])
    if out is None:
        out = torch.empty((N, OH, OW, packed_words(D)), dtype=torch.int64, device=x.device)
    _check(_c().bnn_conv2d_f32_sign(_ptr(x), _ptr(w), N, C, H, W, D, kH, kW, stride[0], stride[1], pad[0], pad[1],
                                     _ptr(scale), _ptr(bias), _ptr(out), _stream()), "bnn_conv2d_f32_sign")
    return out


def bnn_pack_fc_weight_nhwc(w: torch.Tensor, C: int, H: int, W: int) -> torch.Tensor:
    _dev(w, torch.float32, "w")
    assert w.dim() == 2 and w.is_contiguous() and w.shape[1] == C * H * W
    out = torch.empty((w.shape[0], H * W * packed_words(C)), dtype=torch.int64, device=w.device)
    _check(_c().bnn_pack_fc_weight_nhwc(_ptr(w), w.shape[0], C, H, W, _ptr(out), _stream()),
           "bnn_pack_fc_weight_nhwc")
    return out


def bnn_maxpool2x2(a: torch.Tensor, scale: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                   want_int: bool = True, out_i32=None, out_f32=None):
    if (out_i32 is not None or not want_int) and (out_f32 is not None or scale is None):
        st = _t().maxpool(a, out_i32, out_f32, scale, bias)
        if st is not None:
            _check(st, "bnn_maxpool2x2")
            return out_i32, out_f32
    _dev(a, torch.int32, "in")
    assert a.dim() == 4 and a.is_contiguous()
    N, D, H, W = a.shape
    if want_int and out_i32 is None:
        out_i32 = torch.empty((N, D, H // 2, W // 2), dtype=torch.int32, device=a.device)
    if scale is not None and out_f32 is None:
        out_f32 = torch.empty((N, D, H // 2, W // 2), dtype=torch.float32, device=a.device)
    _check(_c().bnn_maxpool2x2(_ptr(a), N, D, H, W, _ptr(out_i32), _ptr(out_f32), _ptr(scale), _ptr(bias),
                                _stream()), "bnn_maxpool2x2")
    return out_i32, out_f32


def bnn_conv2d_f32(x: torch.Tensor, w: torch.Tensor, stride=(1, 1), pad=(0, 0), scale=None, bias=None, out=None):
    if out is not None:
        st = _t().conv2d_f32(x, w, scale, bias, stride, pad, out)
        if st is not None:
            _check(st, "bnn_conv2d_f32")
            return out
    _dev(x, torch.float32, "x")
    _dev(w, torch.float32, "w")
    N, C, H, W = x.shape
    D, _, kH, kW = w.shape
    OH, OW = conv_out_dim(H, kH, stride[0], pad[0]), conv_out_dim(W, kW, stride[1], pad[1])
    if out is None:
        out = torch.empty((N, D, OH, OW), dtype=torch.float32, device=x.device)
    _check(_c().bnn_conv2d_f32(_ptr(x), _ptr(w), N, C, H, W, D, kH, kW, stride[0], stride[1], pad[0], pad[1],
                                _ptr(scale), _ptr(bias), _ptr(out), _stream()), "bnn_conv2d_f32")
    return out


def bnn_fc_f32(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, sign_input: bool = False,
               out=None):
    if out is not None:
        st = _t().fc(x, w, bias, int(sign_input), out)
        if st is not None:
            _check(st, "bnn_fc_f32")
            return out
    _dev(x, torch.float32, "x")
    _dev(w, torch.float32, "w")
    M, K = x.shape
    N = w.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=x.device)
    _check(_c().bnn_fc_f32(_ptr(x), _ptr(w), _ptr(bias), M, K, N, int(sign_input), _ptr(out), _stream()),
           "bnn_fc_f32")
    return out


# ---- 8-bit and gated layers ----------------------------------------------------------
# Gradients come from the backward calls below; torch's autograd does not see these calls, and tensors that require a gradient pass
# without a graph.
FLOATS = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
NORMS = {"none": 0, "rms": 1, "layer": 2}
ACTS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3}


def _float(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda or t.dtype not in FLOATS:
        raise TypeError(f"{name} must be a GPU tensor of dtype {', '.join(map(str, FLOATS))}")
    return FLOATS[t.dtype]


def _rows(t: torch.Tensor, name: str, rows: Optional[int] = None, cols: Optional[int] = None) -> int:
    """The row stride of a matrix (of the given size) whose rows are contiguous."""
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{name}: [{'any' if rows is None else rows}, {'any' if cols is None else cols}] expected, got {list(t.shape)}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the values of a row have to be consecutive")
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0))


def _vector(t: Optional[torch.Tensor], name: str, n: int) -> Optional[int]:
    if t is None:
        return None
    _dev(t, torch.float32, name)
    if t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name}: {n} consecutive values expected")
    return t.data_ptr()


def _workspace(t: torch.Tensor) -> int:
    """Bytes of a workspace that a caller brings; kernels write all through it."""
    if not t.is_cuda:
        raise TypeError("workspace must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError("workspace: a contiguous tensor expected")
    return t.numel() * t.element_size()


def _one_of(table, key, name: str) -> int:
    if key not in table:
        raise ValueError(f"{name}: one of {', '.join(table)}")
    return table[key]


def rows_i8(rows: int, K: int, device="cuda:0") -> torch.Tensor:
    """Room for int8 [rows, K] whose rows start on 16 bytes, which the products read fastest."""
    return torch.empty((rows, (K + 15) // 16 * 16), dtype=torch.int8, device=device)[:, :K]


def bnn_quant_rows_i8(x: torch.Tensor, q: Optional[torch.Tensor] = None,
                      scale: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """x [rows, K] fp32, bf16 or fp16 -> (q int8 [rows, K], scale fp32 [rows])."""
    if q is not None and scale is not None:
        st = _t().quant_rows(x, q, scale)
        if st is not None:
            _check(st, "bnn_quant_rows_i8")
            return q, scale
    kind, ld = _float(x, "x"), _rows(x, "x")
    rows, K = x.shape
    if q is None:
        q = rows_i8(rows, K, x.device)
    if scale is None:
        scale = torch.empty((rows,), dtype=torch.float32, device=x.device)
    _dev(q, torch.int8, "q")
    _check(_c().bnn_quant_rows_i8(_ptr(x), kind, rows, K, ld, _ptr(q), _rows(q, "q", rows, K), _vector(scale, "scale", rows),
                                   _stream()), "bnn_quant_rows_i8")
    return q, scale


def bnn_linear_i8(a: torch.Tensor, a_scale: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor,
                  bias: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                  dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """a int8 [M, K] and its scales [M], b int8 [N, K] and its scales [N] -> [M, N] of out's type, or of dtype."""
    if out is not None:
        st = _t().linear_i8(a, a_scale, b, b_scale, bias, out)
        if st is not None:
            _check(st, "bnn_linear_i8")
            return out
    _dev(a, torch.int8, "a")
    _dev(b, torch.int8, "b")
    lda = _rows(a, "a")
    (M, K), N = a.shape, b.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=dtype, device=a.device)
    _check(_c().bnn_linear_i8(_ptr(a), lda, _vector(a_scale, "a_scale", M), _ptr(b), _rows(b, "b", None, K),
                               _vector(b_scale, "b_scale", N), _vector(bias, "bias", N), M, N, K, _ptr(out),
                               _float(out, "out"), _rows(out, "out", M, N), _stream()), "bnn_linear_i8")
    return out


def _norm_in(b, r, gate, gate_rows, res_scale, w_post, bias_post, w_pre, bias_pre, post, pre, eps) -> NormGateIn:
    r_type, r_ld = _float(r, "r"), _rows(r, "r")
    rows, D = r.shape
    kind, b_ld, gate_ld = r_type, 0, 0
    if b is not None:
        kind, b_ld = _float(b, "b"), _rows(b, "b", rows, D)
    if gate is not None:
        if gate_rows < 1:
            raise ValueError("gate_rows: at least 1")
        _dev(gate, b.dtype if b is not None else r.dtype, "gate")
        gate_ld = _rows(gate, "gate", (rows + gate_rows - 1) // gate_rows, D)
    return NormGateIn(rows, D, kind, r_type, _one_of(NORMS, post, "post"), _one_of(NORMS, pre, "pre"), eps, _ptr(b), b_ld, _ptr(r),
                      r_ld, _ptr(gate), gate_ld, gate_rows if gate is not None else 0, _vector(res_scale, "res_scale", D),
                      _vector(w_post, "w_post", D), _vector(bias_post, "bias_post", D), _vector(w_pre, "w_pre", D),
                      _vector(bias_pre, "bias_pre", D))


def bnn_norm_gate(b: Optional[torch.Tensor], r: torch.Tensor, *, gate: Optional[torch.Tensor] = None, gate_rows: int = 1,
                  res_scale: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None,
                  bias_post: Optional[torch.Tensor] = None, w_pre: Optional[torch.Tensor] = None,
                  bias_pre: Optional[torch.Tensor] = None, post: str = "rms", pre: str = "rms", eps: float = 1e-6,
                  r_out: Optional[torch.Tensor] = None, n_out: Optional[torch.Tensor] = None,
                  q_out: Optional[torch.Tensor] = None, q_scale: Optional[torch.Tensor] = None):
    """b [rows, D] (a block's output, or None before the first), r [rows, D] (the residual stream) -> (r', n): the new stream
    (None without b) and its norm, n_out.  With q_out and q_scale n goes out as int8 rows with scales; n_out is then written
    only if given.  post, pre: "rms", "layer" or "none"."""
    if r_out is None and b is not None:
        r_out = torch.empty(r.shape, dtype=r.dtype, device=r.device)
    if n_out is None and q_out is None and pre != "none":
        n_out = torch.empty(r.shape, dtype=r.dtype if b is None else b.dtype, device=r.device)
    st = _t().norm_gate(b, r, gate, gate_rows, res_scale, w_post, bias_post, w_pre, bias_pre, NORMS.get(post), NORMS.get(pre), eps,
                        r_out, n_out, q_out, q_scale)
    if st is not None:
        _check(st, "bnn_norm_gate")
        return r_out, n_out
    p = _norm_in(b, r, gate, gate_rows, res_scale, w_post, bias_post, w_pre, bias_pre, post, pre, eps)
    rows, D = r.shape
    lds = [0, 0, 0]
    for i, (t, dtype, name) in enumerate(((r_out, r.dtype, "r_out"), (n_out, r.dtype if b is None else b.dtype, "n_out"),
                                          (q_out, torch.int8, "q_out"))):
        if t is not None:
            _dev(t, dtype, name)
            lds[i] = _rows(t, name, rows, D)
    _check(_c().bnn_norm_gate(ctypes.addressof(p), _ptr(r_out), lds[0], _ptr(n_out), lds[1], _ptr(q_out), lds[2],
                               _vector(q_scale, "q_scale", rows), _stream()), "bnn_norm_gate")
    return r_out, n_out


def norm_gate_backward_workspace_bytes(rows: int, D: int, gate_rows: int) -> int:
    return int(_c().bnn_norm_gate_backward_workspace_bytes(rows, D, gate_rows))


NORM_GRADIENTS = ("dr", "db", "dgate", "dres_scale", "dw_post", "dbias_post", "dw_pre", "dbias_pre")


def bnn_norm_gate_backward(b: Optional[torch.Tensor], r: torch.Tensor, dn: Optional[torch.Tensor],
                           dr_out: Optional[torch.Tensor], *, gate: Optional[torch.Tensor] = None, gate_rows: int = 1,
                           res_scale: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None,
                           bias_post: Optional[torch.Tensor] = None, w_pre: Optional[torch.Tensor] = None,
                           bias_pre: Optional[torch.Tensor] = None, post: str = "rms", pre: str = "rms", eps: float = 1e-6,
                           workspace: Optional[torch.Tensor] = None, out=None):
    """Gradients of bnn_norm_gate from its inputs and those of its outputs (dn of n, dr_out of r'; None: zero), as a dict: dr,
    and, for each of b, gate, res_scale, w_post, bias_post, w_pre and bias_pre that was given, its name with a d before it.
    out: the same dict with tensors to write to, where a caller keeps them."""
    if out is None and workspace is None:
        made = _t().norm_gate_gradients(b, r, gate, gate_rows, res_scale, w_post, bias_post, w_pre, bias_pre, NORMS.get(post),
                                        NORMS.get(pre), eps, dn, dr_out)
        if made is not None:
            if type(made) is int:
                _check(made, "bnn_norm_gate_backward")
            return {name: t for name, t in zip(NORM_GRADIENTS, made) if t is not None}
    if workspace is not None:
        _workspace(workspace)
    if r.dim() != 2:
        raise ValueError("r: a matrix expected")
    rows, D = r.shape
    got = dict(out or {})
    wanted = dict(zip(NORM_GRADIENTS, (r, b, gate, res_scale, w_post, bias_post, w_pre, bias_pre)))
    for name, of in wanted.items():
        if of is None:
            got.pop(name, None)
        elif name not in got:
            got[name] = torch.empty(of.shape, dtype=of.dtype, device=r.device)
    if workspace is None:
        nbytes = norm_gate_backward_workspace_bytes(rows, D, gate_rows if gate is not None else 0)
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=r.device)
    st = _t().norm_gate_backward(b, r, gate, gate_rows, res_scale, w_post, bias_post, w_pre, bias_pre, NORMS.get(post), NORMS.get(pre),
                                 eps, dn, dr_out, *[got.get(name) for name in wanted], workspace)
    if st is not None:
        _check(st, "bnn_norm_gate_backward")
        return got
    p = _norm_in(b, r, gate, gate_rows, res_scale, w_post, bias_post, w_pre, bias_pre, post, pre, eps)
    kind = r.dtype if b is None else b.dtype
    mats = [(dn, kind, "dn", rows), (dr_out, r.dtype, "dr_out", rows), (got["dr"], r.dtype, "dr", rows),
            (got.get("db"), kind, "db", rows), (got.get("dgate"), kind, "dgate", gate.shape[0] if gate is not None else 0)]
    args = []
    for t, dtype, name, n in mats:
        if t is not None:
            _dev(t, dtype, name)
        args += [_ptr(t), 0 if t is None else _rows(t, name, n, D)]
    for name in ("dres_scale", "dw_post", "dbias_post", "dw_pre", "dbias_pre"):
        args.append(_vector(got.get(name), name, D))
    _check(_c().bnn_norm_gate_backward(ctypes.addressof(p), *args, _ptr(workspace), _workspace(workspace), _stream()),
           "bnn_norm_gate_backward")
    return got


def gated_ff_saved(T: int, F: int, device="cuda:0") -> torch.Tensor:
    """What bnn_gated_ff leaves for its backward pass, [2, T, F] fp32."""
    return torch.empty((2, T, F), dtype=torch.float32, device=device)


def _saved(saved: torch.Tensor, T: int, F: int) -> int:
    _dev(saved, torch.float32, "saved")
    if tuple(saved.shape) != (2, T, F) or not saved.is_contiguous():
        raise ValueError(f"saved: contiguous [2, {T}, {F}] expected")
    return saved.data_ptr()


def _gated_in(x, wg, wu):
    """(T, D, F, type, strides) of the operands of the two projections."""
    kind, x_ld = _float(x, "x"), _rows(x, "x")
    _dev(wg, x.dtype, "wg")
    _dev(wu, x.dtype, "wu")
    (T, D), F = x.shape, wg.shape[0]
    return T, D, F, kind, (x_ld, _rows(wg, "wg", F, D), _rows(wu, "wu", F, D))


def bnn_gated_ff(x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, act: str = "silu", out: Optional[torch.Tensor] = None,
                 saved: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [T, D], wg and wu [F, D], all bf16 or all fp16 -> h [T, F] = act(x wg^T) * (x wu^T).  act: "silu", "gelu",
    "gelu_tanh" or "relu".  saved (gated_ff_saved): written for bnn_gated_ff_backward."""
    if out is not None:
        st = _t().gated_ff(x, wg, wu, ACTS.get(act), out, saved)
        if st is not None:
            _check(st, "bnn_gated_ff")
            return out
    T, D, F, kind, (x_ld, g_ld, u_ld) = _gated_in(x, wg, wu)
    if out is None:
        out = torch.empty((T, F), dtype=x.dtype, device=x.device)
    _dev(out, x.dtype, "out")
    _check(_c().bnn_gated_ff(_ptr(x), x_ld, _ptr(wg), g_ld, _ptr(wu), u_ld, kind, T, D, F, _one_of(ACTS, act, "act"), _ptr(out),
                              _rows(out, "out", T, F), None if saved is None else _saved(saved, T, F), _stream()), "bnn_gated_ff")
    return out


def bnn_gated_ff_i8(x: torch.Tensor, x_scale: torch.Tensor, wg: torch.Tensor, wg_scale: torch.Tensor, wu: torch.Tensor,
                    wu_scale: torch.Tensor, act: str = "silu", out: Optional[torch.Tensor] = None,
                    dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """bnn_gated_ff on int8 rows with their scales; h of out's type, or of dtype."""
    if out is not None:
        st = _t().gated_ff_i8(x, x_scale, wg, wg_scale, wu, wu_scale, ACTS.get(act), out)
        if st is not None:
            _check(st, "bnn_gated_ff_i8")
            return out
    for t, name in ((x, "x"), (wg, "wg"), (wu, "wu")):
        _dev(t, torch.int8, name)
    x_ld = _rows(x, "x")
    (T, D), F = x.shape, wg.shape[0]
    if out is None:
        out = torch.empty((T, F), dtype=dtype, device=x.device)
    _check(_c().bnn_gated_ff_i8(_ptr(x), x_ld, _vector(x_scale, "x_scale", T), _ptr(wg), _rows(wg, "wg", F, D),
                                 _vector(wg_scale, "wg_scale", F), _ptr(wu), _rows(wu, "wu", F, D), _vector(wu_scale, "wu_scale", F),
                                 T, D, F, _one_of(ACTS, act, "act"), _ptr(out), _float(out, "out"), _rows(out, "out", T, F),
                                 _stream()), "bnn_gated_ff_i8")
    return out


def gated_ff_backward_workspace_bytes(T: int, D: int, F: int) -> int:
    return int(_c().bnn_gated_ff_backward_workspace_bytes(T, D, F))


def bnn_gated_ff_backward(x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, saved: torch.Tensor, dh: torch.Tensor,
                          dx: Optional[torch.Tensor] = None, dwg: Optional[torch.Tensor] = None,
                          dwu: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """(dx, dwg, dwu) from the operands of bnn_gated_ff, what it saved, and dh [T, F]."""
    if dx is None and dwg is None and dwu is None and workspace is None:
        made = _t().gated_ff_gradients(x, wg, wu, saved, dh)
        if made is not None:
            if type(made) is int:
                _check(made, "bnn_gated_ff_backward")
            return made
    if workspace is not None:
        _workspace(workspace)
    if x.dim() != 2 or wg.dim() != 2:
        raise ValueError("x, wg: matrices expected")
    dx, dwg, dwu = (torch.empty(of.shape, dtype=x.dtype, device=x.device) if t is None else t
                    for t, of in ((dx, x), (dwg, wg), (dwu, wu)))
    if workspace is None:
        nbytes = gated_ff_backward_workspace_bytes(x.shape[0], x.shape[1], wg.shape[0])
        workspace = torch.empty(max(16, nbytes), dtype=torch.uint8, device=x.device)
    st = _t().gated_ff_backward(x, wg, wu, saved, dh, dx, dwg, dwu, workspace)
    if st is not None:
        _check(st, "bnn_gated_ff_backward")
        return dx, dwg, dwu
    T, D, F, kind, (x_ld, g_ld, u_ld) = _gated_in(x, wg, wu)
    for t, name in ((dh, "dh"), (dx, "dx"), (dwg, "dwg"), (dwu, "dwu")):
        _dev(t, x.dtype, name)
    _check(_c().bnn_gated_ff_backward(_ptr(x), x_ld, _ptr(wg), g_ld, _ptr(wu), u_ld, kind, T, D, F, _saved(saved, T, F), _ptr(dh),
                                       _rows(dh, "dh", T, F), _ptr(dx), _rows(dx, "dx", T, D), _ptr(dwg), _rows(dwg, "dwg", F, D),
                                       _ptr(dwu), _rows(dwu, "dwu", F, D), _ptr(workspace), _workspace(workspace),
                                       _stream()), "bnn_gated_ff_backward")
    return dx, dwg, dwu


# ---- 8-bit floating point and experts ------------------------------------------------
F8, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
F8_BLOCK = 128


def _present(t: torch.Tensor, name: str, *dtypes: torch.dtype) -> torch.Tensor:
    """A tensor on the current device, whose stream the call goes to."""
    if not t.is_cuda or (dtypes and t.dtype not in dtypes):
        raise TypeError(f"{name} must be a GPU tensor" + (f" of dtype {', '.join(map(str, dtypes))}" if dtypes else ""))
    if t.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on another device than the current one")
    return t


def _float_rows(t: torch.Tensor, name: str, rows: Optional[int] = None, cols: Optional[int] = None) -> Tuple[int, int]:
    """(type, row stride) of a floating-point matrix."""
    _present(t, name, *FLOATS)
    return FLOATS[t.dtype], _rows(t, name, rows, cols)


def _whole(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, *shape: int) -> Optional[int]:
    """A contiguous tensor of this shape, or None."""
    if t is None:
        return None
    _present(t, name, dtype)
    if tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name}: contiguous {list(shape)} expected, got {list(t.shape)}")
    return t.data_ptr()


def _padded(t: torch.Tensor, name: str, shape: Tuple[int, ...], row: int, quantum: int) -> Tuple[int, int, int]:
    """(pointer, row stride, stride between experts) of [.., rows, cols] whose rows have `row` elements of room each."""
    if tuple(t.shape) != shape:
        raise ValueError(f"{name}: {list(shape)} expected, got {list(t.shape)}")
    if shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the values of a row have to be consecutive")
    rows = shape[-2]
    ld = t.stride(-2) if rows > 1 else max((row + quantum - 1) // quantum * quantum, t.stride(-2) // quantum * quantum)
    experts, between = (1, 0) if len(shape) == 2 else (shape[0], t.stride(0))
    if experts == 1:
        between = rows * ld
    if ld < row:
        raise ValueError(f"{name}: rows need room for {row} elements each (rows_f8, scales_f8)")
    if t.numel():
        size = t.element_size()
        last = t.storage_offset() + (experts - 1) * between + (rows - 1) * ld + row
        if t.untyped_storage().nbytes() < last * size:
            raise ValueError(f"{name}: the last row needs room for {row} elements too (rows_f8, scales_f8)")
    return t.data_ptr(), ld, between


def _blocks(K: int) -> int:
    return (K + F8_BLOCK - 1) // F8_BLOCK


def _f8(q: torch.Tensor, scale: torch.Tensor, name: str, shape: Tuple[int, ...]) -> Tuple[int, int, int, int]:
    """Pointers and row strides of rows in e4m3 and of their scales."""
    _present(q, name, F8)
    _present(scale, name + "_scale", E8M0)
    blocks = _blocks(shape[-1])
    pq, ld, _ = _padded(q, name, shape, blocks * F8_BLOCK, 16)
    ps, s_ld, _ = _padded(scale, name + "_scale", (*shape[:-1], blocks), (blocks + 3) // 4 * 4, 4)
    return pq, ld, ps, s_ld


def _f8_weight(b: torch.Tensor, scale: torch.Tensor, name: str, shape: Tuple[int, ...]):
    """((pointer, row stride, stride between experts) of a weight [.., N, K], the same of its scales, their type, rows that share them)."""
    _present(b, name, F8)
    _present(scale, name + "_scale", E8M0, torch.float32)
    N, K = shape[-2:]
    blocks, wide = _blocks(K), scale.dtype == torch.float32
    if scale.dim() != len(shape):
        raise ValueError(f"{name}_scale: {len(shape)} dimensions expected")
    per = 1 if scale.shape[-2] == N and not wide and N > 1 else F8_BLOCK
    room, quantum = (blocks, 1) if wide else ((blocks + 3) // 4 * 4, 4)
    return (_padded(b, name, shape, blocks * F8_BLOCK, 16),
            _padded(scale, name + "_scale", (*shape[:-2], N if per == 1 else _blocks(N), blocks), room, quantum), int(wide), per)


def _made(made, where: str):
    """What a call from the tensors themselves gave, where it was one: its results, or the error of its status."""
    if type(made) is int:
        _check(made, where)
    return made


def rows_f8(rows: int, K: int, device="cuda:0", experts: Optional[int] = None) -> torch.Tensor:
    """Room for e4m3 [rows, K] (or [experts, rows, K]) in rows of whole blocks of 128."""
    lead = (rows,) if experts is None else (experts, rows)
    return torch.empty((*lead, _blocks(K) * F8_BLOCK), dtype=F8, device=device)[..., :K]


def scales_f8(rows: int, K: int, device="cuda:0", experts: Optional[int] = None) -> torch.Tensor:
    """Room for the scales of such rows, one a block: [rows, ceil(K / 128)] (or [experts, rows, ..])."""
    lead = (rows,) if experts is None else (experts, rows)
    return torch.empty((*lead, (_blocks(K) + 3) // 4 * 4), dtype=E8M0, device=device)[..., :_blocks(K)]


def _positions(rows: Optional[torch.Tensor], T: int) -> Tuple[Optional[int], int]:
    if rows is None:
        return None, T
    if rows.dim() != 1:
        raise ValueError("rows: a vector expected")
    return _whole(rows, "rows", torch.int32, rows.shape[0]), rows.shape[0]


def bnn_quant_blocks_f8(x: torch.Tensor, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                        rows: Optional[torch.Tensor] = None, k: int = 1) -> Tuple[torch.Tensor, torch.Tensor]:
    """x [T, K] fp32, bf16 or fp16 -> (q e4m3 [S, K], scale [S, ceil(K / 128)]), powers of two.  rows (bnn_expert_sort): position s is
    x[rows[s] // k], zeros for -1, left as it was for -2; without rows S = T."""
    made = _made(_t().quant_f8(x, q, scale, rows, k, 0), "bnn_quant_blocks_f8")
    if made is not None:
        return made
    kind, ld = _float_rows(x, "x")
    T, K = x.shape
    p_rows, S = _positions(rows, T)
    q = rows_f8(S, K, x.device) if q is None else q
    scale = scales_f8(S, K, x.device) if scale is None else scale
    pq, q_ld, ps, s_ld = _f8(q, scale, "q", (S, K))
    _check(_c().bnn_quant_blocks_f8(_ptr(x), kind, T, ld, p_rows, k, S, K, pq, q_ld, ps, s_ld, _stream()), "bnn_quant_blocks_f8")
    return q, scale


def bnn_quant_columns_f8(x: torch.Tensor, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                         rows: Optional[torch.Tensor] = None, k: int = 1) -> Tuple[torch.Tensor, torch.Tensor]:
    """x [T, D] -> (q e4m3 [D, S], scale [D, ceil(S / 128)]): x, or the rows of it that `rows` names, turned, in blocks along the
    positions; positions without a row are zeros."""
    made = _made(_t().quant_f8(x, q, scale, rows, k, 1), "bnn_quant_columns_f8")
    if made is not None:
        return made
    kind, ld = _float_rows(x, "x")
    T, D = x.shape
    p_rows, S = _positions(rows, T)
    q = rows_f8(D, S, x.device) if q is None else q
    scale = scales_f8(D, S, x.device) if scale is None else scale
    pq, q_ld, ps, s_ld = _f8(q, scale, "q", (D, S))
    _check(_c().bnn_quant_columns_f8(_ptr(x), kind, T, ld, p_rows, k, S, D, pq, q_ld, ps, s_ld, _stream()), "bnn_quant_columns_f8")
    return q, scale


def bnn_quant_weight_f8(w: torch.Tensor, plain: bool = True, turned: bool = True):
    """w [N, K] or [experts, N, K] -> ((q [.., N, K], scale [.., ceil(N / 128), ceil(K / 128)]), the same of w turned), in blocks of 128 x
    128; None for a form that is not wanted."""
    _present(w, "w", *FLOATS)
    if w.dim() not in (2, 3):
        raise ValueError("w: a matrix, or one for each expert")
    if w.shape[-1] > 1 and w.stride(-1) != 1:
        raise ValueError("w: the values of a row have to be consecutive")
    E, (N, K) = None if w.dim() == 2 else w.shape[0], w.shape[-2:]
    made, args = [], []
    for wanted, r, c in ((plain, N, K), (turned, K, N)):
        made.append((rows_f8(r, c, w.device, E), scales_f8(_blocks(r), c, w.device, E)) if wanted else None)
        if wanted:
            q, s = made[-1]
            args.append(F8Weight(_ptr(q), q.stride(-2), 0 if E is None else q.stride(0), _ptr(s), s.stride(-2), 0 if E is None else s.stride(0)))
        else:
            args.append(None)
    ld = w.stride(-2) if N > 1 else max(K, w.stride(-2))
    _check(_c().bnn_quant_weight_f8(_ptr(w), FLOATS[w.dtype], 1 if E is None else E, 0 if E is None else w.stride(0), N, K, ld,
                                     *[None if a is None else ctypes.addressof(a) for a in args], _stream()), "bnn_quant_weight_f8")
    return tuple(made)


FAST_SUMS = 16  # bnn_sums


def bnn_linear_f8(a: torch.Tensor, a_scale: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor,
                  bias: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                  dtype: torch.dtype = torch.bfloat16, fast: bool = False) -> torch.Tensor:
    """a e4m3 [M, K] and its scales, b e4m3 [N, K] and its scales, a row of them for each of its rows or for 128 (these also
    fp32) -> [M, N] of out's type, or of dtype.  fast, here and in the experts' products: bf16 results at up to twice the rate, from sums
    that lose bits (BNN_FAST_SUMS in include/bnn.h)."""
    if out is None and a.dim() == 2 and b.dim() == 2:
        out = torch.empty((a.shape[0], b.shape[0]), dtype=dtype, device=a.device)
    if _made(_t().linear_f8(a, a_scale, b, b_scale, bias, out, FAST_SUMS if fast else 0), "bnn_linear_f8") is not None:
        return out
    if a.dim() != 2 or b.dim() != 2:
        raise ValueError("a, b: matrices expected")
    (M, K), N = a.shape, b.shape[0]
    pa, lda, psa, sa_ld = _f8(a, a_scale, "a", (M, K))
    (pb, ldb, _), (psb, sb_ld, _), wide, per = _f8_weight(b, b_scale, "b", (N, K))
    kind, ldy = _float_rows(out, "out", M, N)
    if bias is not None:
        _present(bias, "bias")
    _check(_c().bnn_linear_f8(pa, lda, psa, sa_ld, pb, ldb, psb, wide, sb_ld, per, _vector(bias, "bias", N), M, N, K, _ptr(out),
                               kind | (FAST_SUMS if fast else 0), ldy, _stream()), "bnn_linear_f8")
    return out


def _offsets(offsets: torch.Tensor, E: int) -> int:
    return _whole(offsets, "offsets", torch.int32, E + 1)


def bnn_expert_linear_f8(a: torch.Tensor, a_scale: torch.Tensor, offsets: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor,
                         out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16, fast: bool = False) -> torch.Tensor:
    """Rows sorted by expert (bnn_expert_sort), a e4m3 [S, K], times their experts' weights, b e4m3 [E, N, K], scales as in
    bnn_linear_f8 -> [S, N]; rows behind the last expert's are left as they were."""
    if out is None and a.dim() == 2 and b.dim() == 3:
        out = torch.empty((a.shape[0], b.shape[1]), dtype=dtype, device=a.device)
    if _made(_t().expert_linear_f8(a, a_scale, offsets, b, b_scale, out, FAST_SUMS if fast else 0), "bnn_expert_linear_f8") is not None:
        return out
    if a.dim() != 2 or b.dim() != 3:
        raise ValueError("a [S, K], b [experts, N, K] expected")
    (S, K), (E, N) = a.shape, b.shape[:2]
    pa, lda, psa, sa_ld = _f8(a, a_scale, "a", (S, K))
    (pb, ldb, b_es), (psb, sb_ld, sb_es), wide, per = _f8_weight(b, b_scale, "b", (E, N, K))
    kind, ldy = _float_rows(out, "out", S, N)
    _check(_c().bnn_expert_linear_f8(pa, lda, psa, sa_ld, _offsets(offsets, E), E, pb, ldb, b_es, psb, wide, sb_ld, sb_es, per, S, N, K,
                                      _ptr(out), kind | (FAST_SUMS if fast else 0), ldy, _stream()), "bnn_expert_linear_f8")
    return out


def bnn_expert_linear_f8_dw(a: torch.Tensor, a_scale: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor, offsets: torch.Tensor,
                            out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.float32, fast: bool = False) -> torch.Tensor:
    """The experts' weights' gradients [E, N, K] from those of the rows, a e4m3 [N, S], and the rows, b e4m3 [K, S], both as
    bnn_quant_columns_f8 gives them; offsets multiples of 128 (bnn_expert_sort with align 128)."""
    if out is None and a.dim() == 2 and b.dim() == 2 and offsets.dim() == 1 and offsets.shape[0] > 0:
        out = torch.empty((offsets.shape[0] - 1, a.shape[0], b.shape[0]), dtype=dtype, device=a.device)
    if _made(_t().expert_linear_f8_dw(a, a_scale, b, b_scale, offsets, out, FAST_SUMS if fast else 0), "bnn_expert_linear_f8_dw") is not None:
        return out
    if a.dim() != 2 or b.dim() != 2 or offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError("a [N, S], b [K, S], offsets [experts + 1] expected")
    (N, S), K, E = a.shape, b.shape[0], offsets.shape[0] - 1
    pa, lda, psa, sa_ld = _f8(a, a_scale, "a", (N, S))
    pb, ldb, psb, sb_ld = _f8(b, b_scale, "b", (K, S))
    _present(out, "out", *FLOATS)
    p_out, ld, es = _padded(out, "out", (E, N, K), K, 1)
    _check(_c().bnn_expert_linear_f8_dw(pa, lda, psa, sa_ld, pb, ldb, psb, sb_ld, _offsets(offsets, E), E, N, K, S, p_out,
                                         FLOATS[out.dtype] | (FAST_SUMS if fast else 0), ld, es, _stream()), "bnn_expert_linear_f8_dw")
    return out


def expert_rows(T: int, k: int, experts: int, align: int = 1) -> int:
    """Positions that the sorted rows of any choices fit into."""
    return int(_c().bnn_expert_rows(T, k, experts, align))


def expert_sort_workspace_bytes(T: int, k: int, experts: int) -> int:
    return int(_c().bnn_expert_sort_workspace_bytes(T, k, experts))


def bnn_expert_sort(experts: torch.Tensor, E: int, align: int = 1, offsets: Optional[torch.Tensor] = None,
                    rows: Optional[torch.Tensor] = None, places: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """experts [T, k] int32 or int64 (outside 0 .. E - 1: none) -> (offsets [E + 1], rows [S], places [T, k]), all int32: where each
    expert's rows begin (multiples of align), the slot token * k + choice at a position, the position of a slot."""
    made = _made(_t().expert_sort(experts, E, align, offsets, rows, places, workspace), "bnn_expert_sort")
    if made is not None:
        return made
    _present(experts, "experts", torch.int32, torch.int64)
    if experts.dim() != 2 or not experts.is_contiguous():
        raise ValueError("experts: contiguous [tokens, choices] expected")
    T, k = experts.shape
    make = dict(dtype=torch.int32, device=experts.device)
    offsets = torch.empty((max(E, 0) + 1,), **make) if offsets is None else offsets
    rows = torch.empty((expert_rows(T, k, E, align),), **make) if rows is None else rows
    places = torch.empty((T, k), **make) if places is None else places
    if workspace is None:
        workspace = torch.empty((expert_sort_workspace_bytes(T, k, E),), dtype=torch.uint8, device=experts.device)
    p_rows, S = _positions(rows, 0)
    _check(_c().bnn_expert_sort(_ptr(experts), experts.element_size(), T, k, E, align, S, _offsets(offsets, E), p_rows,
                                 _whole(places, "places", torch.int32, T, k), _ptr(_present(workspace, "workspace")),
                                 _workspace(workspace), _stream()), "bnn_expert_sort")
    return offsets, rows, places


def bnn_expert_gather(x: torch.Tensor, rows: torch.Tensor, k: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [T, D] -> [S, D]: position s is x[rows[s] // k], zeros for -1, left as it was for -2."""
    made = _made(_t().expert_gather(x, rows, k, out), "bnn_expert_gather")
    if made is not None:
        return made
    kind, ld = _float_rows(x, "x")
    T, D = x.shape
    p_rows, S = _positions(rows, T)
    out = torch.empty((S, D), dtype=x.dtype, device=x.device) if out is None else out
    _present(out, "out", x.dtype)
    _check(_c().bnn_expert_gather(_ptr(x), kind, T, ld, p_rows, k, S, D, _ptr(out), _rows(out, "out", S, D), _stream()), "bnn_expert_gather")
    return out


def bnn_expert_combine(ys: torch.Tensor, places: torch.Tensor, weights: Optional[torch.Tensor] = None,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """ys [S, D] -> [T, D], out[t] = sum over j of weights[t, j] * ys[places[t, j]]; dropped slots (-1) add nothing.  Without weights:
    the gradient of bnn_expert_gather."""
    made = _made(_t().expert_combine(ys, places, weights, out), "bnn_expert_combine")
    if made is not None:
        return made
    kind, ld = _float_rows(ys, "ys")
    (S, D), (T, k) = ys.shape, places.shape
    out = torch.empty((T, D), dtype=ys.dtype, device=ys.device) if out is None else out
    _present(out, "out", ys.dtype)
    _check(_c().bnn_expert_combine(_ptr(ys), kind, S, ld, _whole(places, "places", torch.int32, T, k),
                                    _whole(weights, "weights", torch.float32, T, k), T, k, D, _ptr(out), _rows(out, "out", T, D),
                                    _stream()), "bnn_expert_combine")
    return out


def bnn_expert_combine_backward(ys: torch.Tensor, rows: torch.Tensor, places: torch.Tensor, weights: Optional[torch.Tensor],
                                dout: torch.Tensor, dys: Optional[torch.Tensor] = None,
                                dweights: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(dys [S, D], dweights [T, k]) of bnn_expert_combine from dout [T, D]; positions of no slot between the experts' rows get zeros,
    those behind the last are left as they were."""
    made = _made(_t().expert_combine_backward(ys, rows, places, weights, dout, dys, dweights), "bnn_expert_combine_backward")
    if made is not None:
        return made
    kind, ld = _float_rows(ys, "ys")
    (S, D), (T, k) = ys.shape, places.shape
    p_rows, _ = _positions(rows, S)
    if rows.shape[0] != S:
        raise ValueError(f"rows: {S} positions expected")
    dys = torch.empty((S, D), dtype=ys.dtype, device=ys.device) if dys is None else dys
    dweights = torch.empty((T, k), dtype=torch.float32, device=ys.device) if dweights is None else dweights
    for t, name in ((dout, "dout"), (dys, "dys")):
        _present(t, name, ys.dtype)
    _check(_c().bnn_expert_combine_backward(_ptr(ys), kind, S, ld, p_rows, _whole(places, "places", torch.int32, T, k),
                                             _whole(weights, "weights", torch.float32, T, k), _ptr(dout), _rows(dout, "dout", T, D), T, k,
                                             D, _ptr(dys), _rows(dys, "dys", S, D), _whole(dweights, "dweights", torch.float32, T, k),
                                             _stream()), "bnn_expert_combine_backward")
    return dys, dweights


def _gated(gu: torch.Tensor, act: str, live: Optional[torch.Tensor]):
    kind, ld = _float_rows(gu, "gu")
    if gu.shape[1] % 2:
        raise ValueError("gu: [S, 2 F] expected")
    return gu.shape[0], gu.shape[1] // 2, kind, ld, _one_of(ACTS, act, "act"), _whole(live, "live", torch.int32, 1)


def bnn_gated_act(gu: torch.Tensor, act: str = "silu", out: Optional[torch.Tensor] = None,
                  live: Optional[torch.Tensor] = None) -> torch.Tensor:
    """gu [S, 2 F] = [g | u] -> h [S, F] = act(g) * u.  live (one int32, as offsets[-1:] of bnn_expert_sort): rows from there on are
    left as they were."""
    made = _made(_t().gated_act(gu, ACTS.get(act), out, live), "bnn_gated_act")
    if made is not None:
        return made
    S, F, kind, ld, a, p_live = _gated(gu, act, live)
    out = torch.empty((S, F), dtype=gu.dtype, device=gu.device) if out is None else out
    _present(out, "out", gu.dtype)
    _check(_c().bnn_gated_act(_ptr(gu), kind, S, ld, F, a, p_live, _ptr(out), _rows(out, "out", S, F), _stream()), "bnn_gated_act")
    return out


def bnn_gated_act_f8(gu: torch.Tensor, act: str = "silu", q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                     live: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The same as e4m3 rows with their scales, from h in fp32."""
    made = _made(_t().gated_act_f8(gu, ACTS.get(act), q, scale, live), "bnn_gated_act_f8")
    if made is not None:
        return made
    S, F, kind, ld, a, p_live = _gated(gu, act, live)
    q = rows_f8(S, F, gu.device) if q is None else q
    scale = scales_f8(S, F, gu.device) if scale is None else scale
    pq, q_ld, ps, s_ld = _f8(q, scale, "q", (S, F))
    _check(_c().bnn_gated_act_f8(_ptr(gu), kind, S, ld, F, a, p_live, pq, q_ld, ps, s_ld, _stream()), "bnn_gated_act_f8")
    return q, scale


def bnn_gated_act_backward(gu: torch.Tensor, dh: torch.Tensor, act: str = "silu", out: Optional[torch.Tensor] = None,
                           live: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dgu [S, 2 F] of bnn_gated_act from dh [S, F]."""
    made = _made(_t().gated_act_backward(gu, dh, ACTS.get(act), out, live), "bnn_gated_act_backward")
    if made is not None:
        return made
    S, F, kind, ld, a, p_live = _gated(gu, act, live)
    out = torch.empty((S, 2 * F), dtype=gu.dtype, device=gu.device) if out is None else out
    for t, name in ((dh, "dh"), (out, "out")):
        _present(t, name, gu.dtype)
    _check(_c().bnn_gated_act_backward(_ptr(gu), kind, S, ld, F, a, p_live, _ptr(dh), _rows(dh, "dh", S, F), _ptr(out),
                                        _rows(out, "out", S, 2 * F), _stream()), "bnn_gated_act_backward")
    return out


# ---- measurement helpers (include/bnn_testing.h) -----------------------------------
def prof_enable(on: bool) -> None:
    _check(_c().bnn_prof_enable(int(on)), "bnn_prof_enable")


def prof_reset() -> None:
    _check(_c().bnn_prof_reset(), "bnn_prof_reset")


def prof_records() -> List[Tuple[str, float]]:
    """(kernel name, milliseconds) of every launch recorded since the last reset."""
    L = lib()
    out = []
    kid, ms = _i32(0), ctypes.c_float(0.0)
    for i in range(int(L.bnn_prof_count())):
        _check(L.bnn_prof_get(i, ctypes.byref(kid), ctypes.byref(ms)), "bnn_prof_get")
        out.append((L.bnn_kernel_name(kid.value).decode(), float(ms.value)))
    return out


def bnn_valu_peak_probe(sink: torch.Tensor, blocks: int, iters: int, kind: int = 0) -> None:
    _dev(sink, torch.int32, "sink")
    assert sink.numel() >= blocks * 256
    _check(_c().bnn_valu_peak_probe(_ptr(sink), blocks, iters, kind, _stream()), "bnn_valu_peak_probe")


def bnn_copy_probe(src: torch.Tensor, dst: torch.Tensor) -> None:
    nbytes = src.numel() * src.element_size()
    assert dst.numel() * dst.element_size() >= nbytes
    _check(_c().bnn_copy_probe(_ptr(src), _ptr(dst), nbytes, _stream()), "bnn_copy_probe")

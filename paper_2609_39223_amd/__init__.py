"""Python binding of libqf (C ABI in include/qf.h): argument marshalling only.

Every function takes torch tensors that live on the GPU, passes their device pointers and
the current HIP stream to the C entry point of the same name, and raises ``QFError`` when
the call returns a non-OK status.  All arithmetic runs in the library's HIP kernels; there
is no fallback path.  bf16 tensors may be ``torch.bfloat16`` or raw 16-bit integer tensors.

Tensor conventions follow nn.Linear: X [M, K], W [N, K], Y [M, N]; dW is FP32 [N, K].
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqf.so")

FMT = {"none": 0, "nvfp4": 1, "mxfp4": 2, "q4k": 3}
AMAX_COMPUTE, AMAX_GIVEN = 0, 1
FLAG_REUSE_WS = 1
FLAG_DECODE_IN_GEMM = 2
SCORE = {"softmax": 0, "sigmoid": 1}
STATUS = {0: "QF_OK", 1: "QF_EINVAL", 2: "QF_ESHAPE", 3: "QF_EALIGN", 4: "QF_ENOTSUP",
          5: "QF_EDEVICE"}


class QFError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class QLinearDesc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("ldx", ctypes.c_int64), ("ldw", ctypes.c_int64), ("ldy", ctypes.c_int64),
                ("wfmt", ctypes.c_int32), ("afmt", ctypes.c_int32),
                ("w_amax", ctypes.c_void_p), ("a_amax", ctypes.c_void_p),
                ("flags", ctypes.c_uint32)]


class LoRA(ctypes.Structure):
    _fields_ = [("A", ctypes.c_void_p), ("B", ctypes.c_void_p), ("r", ctypes.c_int64),
                ("scale", ctypes.c_float), ("a_shared", ctypes.c_int32),
                ("b_shared", ctypes.c_int32)]


class Member(ctypes.Structure):
    _fields_ = [("W", ctypes.c_void_p), ("rows", ctypes.c_int64), ("ldw", ctypes.c_int64)]


class PayloadLayout(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_uint64), ("scales", ctypes.c_uint64),
                ("scalars", ctypes.c_uint64), ("total", ctypes.c_uint64)]


class GroupedDesc(ctypes.Structure):
    _fields_ = [("E", ctypes.c_int64), ("T", ctypes.c_int64), ("N", ctypes.c_int64),
                ("K", ctypes.c_int64), ("wfmt", ctypes.c_int32), ("afmt", ctypes.c_int32),
                ("w_amax", ctypes.c_void_p), ("flags", ctypes.c_uint32)]


class Packed(ctypes.Structure):
    _fields_ = [("E", ctypes.c_int64), ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("fmt", ctypes.c_int32), ("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("S", ctypes.c_void_p)]


class KvCache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int64), ("page", ctypes.c_int64), ("H", ctypes.c_int64),
                ("D", ctypes.c_int64), ("fmt", ctypes.c_int32), ("k_codes", ctypes.c_void_p),
                ("k_scales", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p), ("k_S", ctypes.c_void_p), ("v_S", ctypes.c_void_p)]


class KvSeqs(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("offsets", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("table", ctypes.c_void_p), ("cols", ctypes.c_int64), ("max_len", ctypes.c_int64)]


class Adapters(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("r", ctypes.c_int64), ("N", ctypes.c_int64),
                ("K", ctypes.c_int64), ("A", ctypes.c_void_p), ("B", ctypes.c_void_p),
                ("scale", ctypes.c_void_p), ("ranks", ctypes.c_void_p)]


_lib = None
_P = ctypes.c_void_p
_I = ctypes.c_int64


def lib() -> ctypes.CDLL:
    """Load libqf.so (built in-tree by ``__graft_entry__.build()``); no fallback."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build() first")
        torch.cuda.init()  # bind the process's HIP runtime before the library loads
        L = ctypes.CDLL(LIB_PATH)
        sig = {
            "qf_version": ([], ctypes.c_int),
            "qf_last_error": ([], ctypes.c_char_p),
            "qf_amax": ([_P, _I, _I, _I, _P, ctypes.c_int, _P], ctypes.c_int),
            "qf_fakequant_nvfp4": ([_P, _I, _I, _I, _P, ctypes.c_int, _P, _P, _P, _P, _P],
                                   ctypes.c_int),
            "qf_fakequant_mxfp4": ([_P, _I, _I, _I, _P, _P, _P, _P], ctypes.c_int),
            "qf_fakequant_q4k": ([_P, _I, _I, _I, _P, _P, _P], ctypes.c_int),
            "qf_fakequant_q4k_mse": ([_P, _I, _I, _I, _P, _P, _P], ctypes.c_int),
            "qf_workspace_size": ([ctypes.POINTER(QLinearDesc), ctypes.POINTER(ctypes.c_size_t)],
                                  ctypes.c_int),
            "qf_saved_size": ([ctypes.POINTER(QLinearDesc), ctypes.POINTER(ctypes.c_size_t)],
                              ctypes.c_int),
            "qf_qlinear_fwd": ([ctypes.POINTER(QLinearDesc), _P, _P, _P, _P, _P, ctypes.c_size_t,
                                _P], ctypes.c_int),
            "qf_qlinear_fwd_noalloc": ([ctypes.POINTER(QLinearDesc), _P, _P, _P, _P],
                                       ctypes.c_int),
            "qf_qlinear_bwd_ste": ([ctypes.POINTER(QLinearDesc), _P, _P, _P, _P, _P, _P, _P,
                                    ctypes.c_size_t, _P], ctypes.c_int),
            "qf_fragment_bytes": ([_I, _I, ctypes.POINTER(ctypes.c_size_t)], ctypes.c_int),
            "qf_pack_fragments": ([_P, _I, _I, _I, _P, _P], ctypes.c_int),
            "qf_gemm_bf16_fragb": ([_I, _I, _I, _P, _I, _P, _P, _I, ctypes.c_int, _P,
                                    ctypes.c_size_t, _P], ctypes.c_int),
            "qf_gemm_packed_b": ([_I, _I, _I, _P, _I, ctypes.c_int, _P, _P, _P, _P, _I, _P],
                                 ctypes.c_int),
            "qf_dequantize_transposed": ([ctypes.c_int, _P, _P, _P, _I, _I, _P, _I, _P],
                                         ctypes.c_int),
            "qf_validate_fakequant": ([ctypes.c_int, _P, _I, _I, _I], ctypes.c_int),
            "qf_validate_qlinear": ([ctypes.POINTER(QLinearDesc), _P, _P, _P, _P, _P,
                                     ctypes.c_size_t], ctypes.c_int),
            "qf_validate_grouped": ([ctypes.POINTER(GroupedDesc), _P, _P, _P, _P, _P,
                                     ctypes.c_size_t], ctypes.c_int),
            "qf_grouped_workspace_size": ([ctypes.POINTER(GroupedDesc),
                                           ctypes.POINTER(ctypes.c_size_t)], ctypes.c_int),
            "qf_grouped_saved_size": ([ctypes.POINTER(GroupedDesc),
                                       ctypes.POINTER(ctypes.c_size_t)], ctypes.c_int),
            "qf_qlinear_grouped_fwd": ([ctypes.POINTER(GroupedDesc), _P, _P, _P, _P, _P, _P,
                                        ctypes.c_size_t, _P], ctypes.c_int),
            "qf_qlinear_grouped_bwd_ste": ([ctypes.POINTER(GroupedDesc), _P, _P, _P, _P, _P, _P,
                                            _P, _P, ctypes.c_size_t, _P], ctypes.c_int),
            "qf_gemm_bf16": ([_I, _I, _I, _P, _I, ctypes.c_int, _P, _I, ctypes.c_int, _P, _I,
                              ctypes.c_int, _P], ctypes.c_int),
            "qf_transpose_bf16": ([_P, _I, _I, _I, _P, _I, _P], ctypes.c_int),
            "qf_gemm_workspace_size": ([_I, _I, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)],
                                       ctypes.c_int),
            "qf_gemm_bf16_ws": ([_I, _I, _I, _P, _I, ctypes.c_int, _P, _I, ctypes.c_int, _P, _I,
                                 ctypes.c_int, _P, ctypes.c_size_t, _P], ctypes.c_int),
            "qf_gemm_bf16_at": ([_I, _I, _I, _P, _I, _P, _I, _P, _I, _P, _I, _P], ctypes.c_int),
            "qf_fakequant_transposed": ([ctypes.c_int, _P, _I, _I, _I, _P, _P, _I, _P],
                                        ctypes.c_int),
            "qf_lora_amax": ([_P, _I, _I, _I, ctypes.POINTER(LoRA), _P, ctypes.c_int, _P],
                             ctypes.c_int),
            "qf_lora_fakequant": ([ctypes.c_int, _P, _I, _I, _I, ctypes.POINTER(LoRA), _P,
                                   ctypes.c_int, _P, _P, _P, _P, _P, _P], ctypes.c_int),
            "qf_lora_fakequant_transposed": ([ctypes.c_int, _P, _I, _I, _I, ctypes.POINTER(LoRA),
                                              _P, _P, _I, _P], ctypes.c_int),
            "qf_lora_workspace_size": ([ctypes.POINTER(QLinearDesc), ctypes.POINTER(LoRA),
                                        ctypes.POINTER(ctypes.c_size_t)], ctypes.c_int),
            "qf_qlinear_lora_fwd": ([ctypes.POINTER(QLinearDesc), ctypes.POINTER(LoRA), _P, _P,
                                     _P, _P, ctypes.c_size_t, _P], ctypes.c_int),
            "qf_qlinear_lora_bwd_ste": ([ctypes.POINTER(QLinearDesc), ctypes.POINTER(LoRA), _P,
                                         _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P],
                                        ctypes.c_int),
            "qf_qad_kl": ([_P, _I, _P, _I, _I, _I, ctypes.c_float, _P, _P, _P, _I, _P, _P],
                          ctypes.c_int),
            "qf_export_fused": ([ctypes.c_int, ctypes.POINTER(Member), ctypes.c_int, _I, _P, _P,
                                 _P, _P, _P, _P, _P], ctypes.c_int),
            "qf_payload_layout_of": ([ctypes.c_int, _I, _I, ctypes.POINTER(PayloadLayout)],
                                     ctypes.c_int),
            "qf_payload_write_header": ([ctypes.c_int, _I, _I, _P, _P], ctypes.c_int),
            "qf_grouped_lora_workspace_size": ([ctypes.POINTER(GroupedDesc), ctypes.POINTER(LoRA),
                                                ctypes.POINTER(ctypes.c_size_t)], ctypes.c_int),
            "qf_qlinear_grouped_lora_fwd": ([ctypes.POINTER(GroupedDesc), ctypes.POINTER(LoRA), _P,
                                             _P, _P, _P, _P, ctypes.c_size_t, _P], ctypes.c_int),
            "qf_qlinear_grouped_lora_bwd_ste": ([ctypes.POINTER(GroupedDesc), ctypes.POINTER(LoRA),
                                                 _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t,
                                                 _P], ctypes.c_int),
            "qf_moe_route": ([_P, ctypes.c_int, _I, _I, _I, _I, ctypes.c_int, ctypes.c_int,
                              ctypes.c_float, _P, _P, _P, _P], ctypes.c_int),
            "qf_moe_route_bwd": ([_P, ctypes.c_int, _I, _I, _I, _I, ctypes.c_int, ctypes.c_int,
                                  ctypes.c_float, _P, _P, _P, _I, _P], ctypes.c_int),
            "qf_moe_dispatch_workspace_size": ([_I, _I, _I, ctypes.POINTER(ctypes.c_size_t)],
                                               ctypes.c_int),
            "qf_moe_dispatch": ([_P, _I, _I, _I, _P, _P, _P, _P, _I, _I, _P, _P, ctypes.c_size_t,
                                 _P], ctypes.c_int),
            "qf_moe_dispatch_bwd": ([_P, _I, _I, _I, _P, _P, _I, _P], ctypes.c_int),
            "qf_moe_combine": ([_P, _P, _I, _I, _I, _P, _P, _I, _P], ctypes.c_int),
            "qf_moe_combine_bwd": ([_P, _P, _I, _I, _I, _P, _I, _P, _P, _P, _P], ctypes.c_int),
            "qf_packed_matvec": ([ctypes.POINTER(Packed), _I, _P, _I, _P, _I, ctypes.c_int, _P],
                                 ctypes.c_int),
            "qf_packed_matvec_grouped": ([ctypes.POINTER(Packed), _P, _I, _P, _I, _I, _P, _I, _P, _I,
                                          ctypes.c_int, _P], ctypes.c_int),
            "qf_kv_write": ([ctypes.POINTER(KvCache), ctypes.POINTER(KvSeqs), _I, _P, _I, _P, _I, _P],
                            ctypes.c_int),
            "qf_kv_read": ([ctypes.POINTER(KvCache), ctypes.POINTER(KvSeqs), _I, _P, _I, _P, _I, _P],
                           ctypes.c_int),
            "qf_kv_attention_workspace_size": ([ctypes.POINTER(KvCache), ctypes.POINTER(KvSeqs), _I, _I,
                                                _I, ctypes.POINTER(ctypes.c_size_t)], ctypes.c_int),
            "qf_kv_attention": ([ctypes.POINTER(KvCache), ctypes.POINTER(KvSeqs), _I, _P, _I, _I,
                                 ctypes.c_float, _I, _P, _I, _P, _P, ctypes.c_size_t, _P], ctypes.c_int),
            "qf_lora_rows_workspace_size": ([ctypes.POINTER(Adapters), _I,
                                             ctypes.POINTER(ctypes.c_size_t)], ctypes.c_int),
            "qf_lora_rows": ([ctypes.POINTER(Adapters), _P, _I, _P, _I, _P, _I, _P, _I, ctypes.c_int, _P,
                              ctypes.c_size_t, _P], ctypes.c_int),
        }
        for name, (args, res) in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        _lib = L
    return _lib


def _check(status: int):
    if status != 0:
        raise QFError(status, lib().qf_last_error().decode())


def _ptr(t):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError("expected a torch.Tensor")
    if not t.is_cuda:
        raise ValueError("tensor must be on the GPU")
    return t.data_ptr()


def _stream():
    # the handle alone: building the Stream object around it takes 2.9 us of host time, this 0.6
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _bf16(t):
    if t is not None and t.element_size() != 2:
        raise TypeError("bf16 operand must have 2-byte elements")
    return t


def _rows(x):
    if x.dim() != 2:
        raise ValueError("expected a 2-D tensor")
    if x.stride(1) != 1:
        raise ValueError("rows must be contiguous")
    return x.shape[0], x.shape[1], x.stride(0)


def version() -> int:
    return lib().qf_version()


# ----------------------------------------------------------------------------- quantizers
def amax(x, out, accumulate: bool = False):
    R, K, ld = _rows(_bf16(x))
    _check(lib().qf_amax(_ptr(x), R, K, ld, _ptr(out), int(accumulate), _stream()))
    return out


def fakequant_nvfp4(x, amax, amax_mode=AMAX_COMPUTE, s_out=None, codes=None, scales=None,
                    xhat=None):
    R, K, ld = _rows(_bf16(x))
    _check(lib().qf_fakequant_nvfp4(_ptr(x), R, K, ld, _ptr(amax), int(amax_mode), _ptr(s_out),
                                    _ptr(codes), _ptr(scales), _ptr(xhat), _stream()))


def fakequant_mxfp4(x, codes=None, scales=None, xhat=None):
    R, K, ld = _rows(_bf16(x))
    _check(lib().qf_fakequant_mxfp4(_ptr(x), R, K, ld, _ptr(codes), _ptr(scales), _ptr(xhat),
                                    _stream()))


def fakequant_q4k(x, packed=None, xhat=None):
    R, K, ld = _rows(_bf16(x))
    _check(lib().qf_fakequant_q4k(_ptr(x), R, K, ld, _ptr(packed), _ptr(xhat), _stream()))


def fakequant_q4k_mse(x, packed=None, xhat=None):
    R, K, ld = _rows(_bf16(x))
    _check(lib().qf_fakequant_q4k_mse(_ptr(x), R, K, ld, _ptr(packed), _ptr(xhat), _stream()))


def fakequant_transposed(x, fmt, out, amax=None):
    """out[k][r] = x_hat[r][k] for x [R, K]; out is a [K, >=R] row-contiguous bf16 tensor."""
    R, K, ld = _rows(_bf16(x))
    if out.dim() != 2 or out.shape[0] != K or out.shape[1] < R or out.stride(1) != 1:
        raise ValueError("out must be a [K, >=R] row-contiguous tensor")
    _check(lib().qf_fakequant_transposed(FMT[fmt], _ptr(x), R, K, ld, _ptr(amax),
                                         _ptr(_bf16(out)), out.stride(0), _stream()))
    return out


# --------------------------------------------------------------------------- linear layer
def qlinear_desc(M, N, K, wfmt="nvfp4", afmt="none", w_amax=None, a_amax=None, flags=0,
                 ldx=0, ldw=0, ldy=0) -> QLinearDesc:
    return QLinearDesc(M, N, K, ldx, ldw, ldy, FMT[wfmt], FMT[afmt], _ptr(w_amax),
                       _ptr(a_amax), flags)


def workspace_size(desc: QLinearDesc) -> int:
    n = ctypes.c_size_t()
    _check(lib().qf_workspace_size(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def workspace(desc: QLinearDesc, device="cuda"):
    return torch.empty(max(workspace_size(desc), 256), dtype=torch.uint8, device=device)


def saved_size(desc: QLinearDesc) -> int:
    n = ctypes.c_size_t()
    _check(lib().qf_saved_size(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def saved_buffer(desc: QLinearDesc, device="cuda"):
    """A device buffer for the layer's saved (packed) operands, qf_saved_size bytes."""
    return torch.empty(max(saved_size(desc), 256), dtype=torch.uint8, device=device)


def qlinear_fwd(desc, X, W, Y, ws, saved=None):
    _check(lib().qf_qlinear_fwd(ctypes.byref(desc), _ptr(_bf16(X)), _ptr(_bf16(W)),
                                _ptr(_bf16(Y)), _ptr(saved), _ptr(ws), ws.numel(), _stream()))
    return Y


def qlinear_fwd_noalloc(desc, X, W, Y):
    """qf_qlinear_fwd_noalloc: the forward with the library's static device scratch."""
    _check(lib().qf_qlinear_fwd_noalloc(ctypes.byref(desc), _ptr(_bf16(X)), _ptr(_bf16(W)),
                                        _ptr(_bf16(Y)), _stream()))
    return Y


def qlinear_bwd_ste(desc, dY, X, W, dX, dW, ws, saved=None):
    _check(lib().qf_qlinear_bwd_ste(ctypes.byref(desc), _ptr(_bf16(dY)), _ptr(_bf16(X)),
                                    _ptr(_bf16(W)), _ptr(saved), _ptr(_bf16(dX)), _ptr(dW),
                                    _ptr(ws), ws.numel(), _stream()))


def grouped_desc(E, T, N, K, wfmt="nvfp4", afmt="none", w_amax=None, flags=0) -> GroupedDesc:
    return GroupedDesc(E, T, N, K, FMT[wfmt], FMT[afmt], _ptr(w_amax), flags)


def grouped_workspace(desc: GroupedDesc, device="cuda"):
    n = ctypes.c_size_t()
    _check(lib().qf_grouped_workspace_size(ctypes.byref(desc), ctypes.byref(n)))
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def grouped_saved_size(desc: GroupedDesc) -> int:
    n = ctypes.c_size_t()
    _check(lib().qf_grouped_saved_size(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def grouped_saved_buffer(desc: GroupedDesc, device="cuda"):
    """A device buffer for the grouped layer's saved operand (the experts' packed W_hat)."""
    return torch.empty(max(grouped_saved_size(desc), 256), dtype=torch.uint8, device=device)


def qlinear_grouped_fwd(desc, offsets, X, W, Y, ws, saved=None):
    _check(lib().qf_qlinear_grouped_fwd(ctypes.byref(desc), _ptr(offsets), _ptr(_bf16(X)),
                                        _ptr(_bf16(W)), _ptr(_bf16(Y)), _ptr(saved), _ptr(ws),
                                        ws.numel(), _stream()))


def qlinear_grouped_bwd_ste(desc, offsets, dY, X, W, dX, dW, ws, saved=None):
    _check(lib().qf_qlinear_grouped_bwd_ste(ctypes.byref(desc), _ptr(offsets), _ptr(_bf16(dY)),
                                            _ptr(_bf16(X)), _ptr(_bf16(W)), _ptr(saved),
                                            _ptr(_bf16(dX)), _ptr(dW), _ptr(ws), ws.numel(),
                                            _stream()))


def gemm_bf16(M, N, K, A, lda, a_kmajor, B, ldb, b_kmajor, C, ldc, c_f32, ws=None):
    if ws is None:
        _check(lib().qf_gemm_bf16(M, N, K, _ptr(_bf16(A)), lda, int(a_kmajor), _ptr(_bf16(B)),
                                  ldb, int(b_kmajor), _ptr(C), ldc, int(c_f32), _stream()))
    else:
        _check(lib().qf_gemm_bf16_ws(M, N, K, _ptr(_bf16(A)), lda, int(a_kmajor), _ptr(_bf16(B)),
                                     ldb, int(b_kmajor), _ptr(C), ldc, int(c_f32), _ptr(ws),
                                     ws.numel() * ws.element_size(), _stream()))
    return C


def gemm_bf16_at(M, N, K, A, lda, B, ldb, C, ldc, at, ldat):
    _check(lib().qf_gemm_bf16_at(M, N, K, _ptr(_bf16(A)), lda, _ptr(_bf16(B)), ldb,
                                 _ptr(_bf16(C)), ldc, _ptr(_bf16(at)), ldat, _stream()))
    return C, at


def fragment_bytes(N, K) -> int:
    n = ctypes.c_size_t()
    _check(lib().qf_fragment_bytes(N, K, ctypes.byref(n)))
    return n.value


def pack_fragments(B, out):
    """qf_pack_fragments: out (a flat 16-bit tensor of fragment_bytes(N, K) bytes) from B [N, K]."""
    N, K, ld = _rows(_bf16(B))
    _check(lib().qf_pack_fragments(_ptr(_bf16(B)), N, K, ld, _ptr(out), _stream()))
    return out


def gemm_bf16_fragb(M, N, K, A, lda, Bf, C, ldc, c_f32, ws=None):
    """qf_gemm_bf16_fragb: C = A B^T with B in the fragment-major layout."""
    _check(lib().qf_gemm_bf16_fragb(M, N, K, _ptr(_bf16(A)), lda, _ptr(Bf), _ptr(C), ldc,
                                    int(c_f32), _ptr(ws), 0 if ws is None else ws.numel(),
                                    _stream()))
    return C


def gemm_packed_b(M, N, K, A, lda, fmt, codes, scales, S, C, ldc):
    """qf_gemm_packed_b: C = A W_hat^T with W_hat decoded inside the GEMM from packed codes."""
    _check(lib().qf_gemm_packed_b(M, N, K, _ptr(_bf16(A)), lda, FMT[fmt], _ptr(codes),
                                  _ptr(scales), _ptr(S), _ptr(_bf16(C)), ldc, _stream()))
    return C


def dequantize_transposed(fmt, codes, scales, S, R, K, out):
    """qf_dequantize_transposed: out[k][r] = x_hat[r][k] from packed codes (out [K, >=R])."""
    if out.dim() != 2 or out.shape[0] != K or out.shape[1] < R or out.stride(1) != 1:
        raise ValueError("out must be a [K, >=R] row-contiguous tensor")
    _check(lib().qf_dequantize_transposed(FMT[fmt], _ptr(codes), _ptr(scales), _ptr(S), R, K,
                                          _ptr(_bf16(out)), out.stride(0), _stream()))
    return out


def gemm_workspace(M, N, c_f32, device="cuda"):
    n = ctypes.c_size_t()
    _check(lib().qf_gemm_workspace_size(M, N, int(c_f32), ctypes.byref(n)))
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def transpose_bf16(x, out):
    """out[c][r] = x[r][c] (bf16, R and C multiples of 8)."""
    R, C, ld = _rows(_bf16(x))
    if out.dim() != 2 or out.shape[0] != C or out.shape[1] < R or out.stride(1) != 1:
        raise ValueError("out must be a [C, >=R] row-contiguous tensor")
    _check(lib().qf_transpose_bf16(_ptr(x), R, C, ld, _ptr(_bf16(out)), out.stride(0), _stream()))
    return out


# --------------------------------------------------------------------------- LoRA-QAD
def lora(A, B, scale=1.0, a_shared=False, b_shared=False) -> LoRA:
    """Adapter descriptor: A FP32 [r, K] (or [E, r, K]), B FP32 [N, r] (or [E, N, r]).
    The descriptor holds references to A and B, so the device memory it points to stays
    allocated while the descriptor is alive."""
    for t in (A, B):
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise TypeError("LoRA factors must be contiguous float32 tensors")
    r = A.shape[-2]
    if B.shape[-1] != r:
        raise ValueError("A is [.., r, K] and B is [.., N, r]")
    lo = LoRA(_ptr(A), _ptr(B), r, float(scale), int(a_shared), int(b_shared))
    lo._factors = (A, B)
    return lo


def lora_amax(W, lo: LoRA, out, accumulate: bool = False):
    N, K, ld = _rows(_bf16(W))
    _check(lib().qf_lora_amax(_ptr(W), N, K, ld, ctypes.byref(lo), _ptr(out), int(accumulate),
                              _stream()))
    return out


def lora_fakequant(W, lo: LoRA, fmt, amax=None, amax_mode=AMAX_COMPUTE, s_out=None, codes=None,
                   scales=None, packed=None, xhat=None):
    N, K, ld = _rows(_bf16(W))
    _check(lib().qf_lora_fakequant(FMT[fmt], _ptr(W), N, K, ld, ctypes.byref(lo), _ptr(amax),
                                   amax_mode, _ptr(s_out), _ptr(codes), _ptr(scales),
                                   _ptr(packed), _ptr(_bf16(xhat)), _stream()))


def lora_fakequant_transposed(W, lo: LoRA, fmt, out, amax=None):
    N, K, ld = _rows(_bf16(W))
    if out.dim() != 2 or out.shape[0] != K or out.shape[1] < N or out.stride(1) != 1:
        raise ValueError("out must be a [K, >=N] row-contiguous tensor")
    _check(lib().qf_lora_fakequant_transposed(FMT[fmt], _ptr(W), N, K, ld, ctypes.byref(lo),
                                              _ptr(amax), _ptr(_bf16(out)), out.stride(0),
                                              _stream()))
    return out


def lora_workspace(desc: QLinearDesc, lo: LoRA, device="cuda"):
    n = ctypes.c_size_t()
    _check(lib().qf_lora_workspace_size(ctypes.byref(desc), ctypes.byref(lo), ctypes.byref(n)))
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def qlinear_lora_fwd(desc, lo: LoRA, X, W, Y, ws):
    _check(lib().qf_qlinear_lora_fwd(ctypes.byref(desc), ctypes.byref(lo), _ptr(_bf16(X)),
                                     _ptr(_bf16(W)), _ptr(_bf16(Y)), _ptr(ws), ws.numel(),
                                     _stream()))
    return Y


def qlinear_lora_bwd_ste(desc, lo: LoRA, dY, X, W, dX, dA, dB, ws):
    _check(lib().qf_qlinear_lora_bwd_ste(ctypes.byref(desc), ctypes.byref(lo), _ptr(_bf16(dY)),
                                         _ptr(_bf16(X)), _ptr(_bf16(W)), _ptr(_bf16(dX)),
                                         _ptr(dA), _ptr(dB), _ptr(ws), ws.numel(), _stream()))


def grouped_lora_workspace(desc: GroupedDesc, lo: LoRA, device="cuda"):
    n = ctypes.c_size_t()
    _check(lib().qf_grouped_lora_workspace_size(ctypes.byref(desc), ctypes.byref(lo),
                                                ctypes.byref(n)))
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def qlinear_grouped_lora_fwd(desc, lo: LoRA, offsets, X, W, Y, ws):
    _check(lib().qf_qlinear_grouped_lora_fwd(ctypes.byref(desc), ctypes.byref(lo), _ptr(offsets),
                                             _ptr(_bf16(X)), _ptr(_bf16(W)), _ptr(_bf16(Y)),
                                             _ptr(ws), ws.numel(), _stream()))


def qlinear_grouped_lora_bwd_ste(desc, lo: LoRA, offsets, dY, X, W, dX, dA, dB, ws):
    _check(lib().qf_qlinear_grouped_lora_bwd_ste(ctypes.byref(desc), ctypes.byref(lo),
                                                 _ptr(offsets), _ptr(_bf16(dY)), _ptr(_bf16(X)),
                                                 _ptr(_bf16(W)), _ptr(_bf16(dX)), _ptr(dA),
                                                 _ptr(dB), _ptr(ws), ws.numel(), _stream()))


# ---------------------------------------------------- around the grouped layer (MoE)
def _mat(x):
    """_rows for operands that may be empty or a single row, whose row stride means nothing."""
    st = x.stride()
    if len(st) != 2:
        raise ValueError("expected a 2-D tensor")
    R, C = x.shape
    if R > 1 and C > 1:
        if st[1] != 1:
            raise ValueError("rows must be contiguous")
        return R, C, st[0]
    if C > 1 and R == 1 and st[1] != 1:
        raise ValueError("rows must be contiguous")
    return R, C, st[0] if R > 1 and C else (C + 7) // 8 * 8


def _typed(t, dtype, name, shape=None):
    """t must be a contiguous tensor of the given type (and shape); None passes."""
    if t is not None:
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if shape is not None and t.shape != shape:
            raise ValueError(f"{name} must be {shape}, not {tuple(t.shape)}")
    return _ptr(t)


def _logits(z):
    T, E, ld = _mat(z)
    if z.dtype == torch.float32:
        return T, E, ld, 1
    _bf16(z)
    return T, E, ld, 0


def moe_route(z, ids, w, score="softmax", norm=True, scale=1.0, mask=None):
    """The ids.shape[1] largest logits of every row of z [T, E] (ids int32, w float32 [T, k]); mask: bool
    or uint8 [T], false for padding."""
    T, E, ld, f32 = _logits(z)
    k = ids.shape[1]
    if mask is not None and mask.dtype == torch.bool:
        mask = mask.view(torch.uint8)
    _check(lib().qf_moe_route(_ptr(z), f32, T, E, ld, k, SCORE[score], int(norm), float(scale),
                              _typed(mask, torch.uint8, "mask", (T,)),
                              _typed(ids, torch.int32, "ids", (T, k)),
                              _typed(w, torch.float32, "w", (T, k)), _stream()))
    return ids, w


def moe_route_bwd(z, ids, dw, dz, score="softmax", norm=True, scale=1.0):
    """dz [T, E], of z's type, from dw float32 [T, k] and the forward's z and ids."""
    T, E, ld, f32 = _logits(z)
    T2, E2, lddz, f2 = _logits(dz)
    if (T2, E2, f2) != (T, E, f32):
        raise ValueError("dz must have the shape and type of z")
    k = ids.shape[1]
    _check(lib().qf_moe_route_bwd(_ptr(z), f32, T, E, ld, k, SCORE[score], int(norm), float(scale),
                                  _typed(ids, torch.int32, "ids", (T, k)),
                                  _typed(dw, torch.float32, "dw", (T, k)), _ptr(dz), lddz,
                                  _stream()))
    return dz


def moe_dispatch_workspace(T, E, k, device="cuda"):
    n = ctypes.c_size_t()
    _check(lib().qf_moe_dispatch_workspace_size(T, E, k, ctypes.byref(n)))
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def moe_dispatch(ids, offsets, row_of, slot_of, ws, X=None, Xg=None):
    """Stable sort of the slots of ids [T, k] by expert (offsets int64 [E+1], row_of int32 [T, k],
    slot_of int32 [T k]) and, with X [T, H], its rows in that order (Xg [T k, H])."""
    T, k = ids.shape
    H = ldx = 0
    if X is not None and Xg is not None:
        R, H, ldx = _mat(_bf16(X))
        if R != T:
            raise ValueError("X must have a row for every token")
        _typed(_bf16(Xg), Xg.dtype, "Xg", (T * k, H))
    _check(lib().qf_moe_dispatch(_typed(ids, torch.int32, "ids"), T, offsets.numel() - 1, k,
                                 _typed(offsets, torch.int64, "offsets"),
                                 _typed(row_of, torch.int32, "row_of", (T, k)),
                                 _typed(slot_of, torch.int32, "slot_of", (T * k,)), _ptr(X), H, ldx,
                                 _ptr(Xg), _ptr(ws), ws.numel(), _stream()))
    return offsets, row_of, slot_of


def _grouped_rows(g, name, T, k, H):
    return _typed(_bf16(g), g.dtype if g is not None else None, name, (T * k, H))


def moe_dispatch_bwd(row_of, dXg, dX):
    """dX[t] = sum over j of dXg[row_of[t, j]]."""
    T, k = row_of.shape
    R, H, ld = _mat(_bf16(dX))
    if R != T:
        raise ValueError("dX must have a row for every token")
    _check(lib().qf_moe_dispatch_bwd(_typed(row_of, torch.int32, "row_of"), T, k, H,
                                     _grouped_rows(dXg, "dXg", T, k, H), _ptr(dX), ld, _stream()))
    return dX


def moe_combine(row_of, Yg, Y, w=None):
    """Y[t] = sum over j of w[t, j] Yg[row_of[t, j]] (w None: ones)."""
    T, k = row_of.shape
    R, H, ld = _mat(_bf16(Y))
    if R != T:
        raise ValueError("Y must have a row for every token")
    _check(lib().qf_moe_combine(_typed(row_of, torch.int32, "row_of"),
                                _typed(w, torch.float32, "w", (T, k)), T, k, H,
                                _grouped_rows(Yg, "Yg", T, k, H), _ptr(Y), ld, _stream()))
    return Y


def moe_combine_bwd(row_of, dY, dYg, Yg=None, w=None, dw=None):
    """dYg[row_of[t, j]] = w[t, j] dY[t] and dw[t, j] = <dY[t], Yg[row_of[t, j]]>."""
    T, k = row_of.shape
    R, H, ld = _mat(_bf16(dY))
    if R != T:
        raise ValueError("dY must have a row for every token")
    _check(lib().qf_moe_combine_bwd(_typed(row_of, torch.int32, "row_of"),
                                    _typed(w, torch.float32, "w", (T, k)), T, k, H, _ptr(dY), ld,
                                    _grouped_rows(Yg, "Yg", T, k, H),
                                    _grouped_rows(dYg, "dYg", T, k, H),
                                    _typed(dw, torch.float32, "dw", (T, k)), _stream()))


# ---------------------------------------------------- few rows times packed weights
def packed_weight(fmt, N, K, codes, scales=None, S=None, E=None) -> Packed:
    """Descriptor of one packed weight [N, K] (E None) or of E of them back to back: codes, block
    scales and (NVFP4) float32 tensor scales as the quantizers write them.  It holds references to
    the tensors, so their device memory stays allocated while the descriptor is alive."""
    n, block = (1 if E is None else E) * N, {"nvfp4": 16, "mxfp4": 32, "q4k": 256}[fmt]
    if K % block == 0:
        for t, name, size in ((codes, "codes", n * K // 256 * 144 if fmt == "q4k" else n * K // 2),
                              (scales, "scales", 0 if fmt == "q4k" else n * K // block)):
            if t is not None and size and t.numel() * t.element_size() < size:
                raise ValueError(f"{name} holds fewer than {size} bytes")
        if fmt == "nvfp4" and S is not None and S.numel() < (1 if E is None else E):
            raise ValueError("S needs a tensor scale for every weight")
    for t, name in ((codes, "codes"), (scales, "scales")):
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    p = Packed(1 if E is None else E, N, K, FMT[fmt], _ptr(codes), _ptr(scales),
               _typed(S, torch.float32, "S"))
    p._tensors = (codes, scales, S)
    return p


def _products(Y):
    R, N, ld = _mat(Y)
    if Y.dtype == torch.float32:
        return R, N, ld, 1
    _bf16(Y)
    return R, N, ld, 0


def packed_matvec(weight: Packed, X, Y):
    """Y [M, N] (bf16 or float32) = X W^T for up to 64 rows of X."""
    M, K, ldx = _mat(_bf16(X))
    R, N, ldy, f32 = _products(Y)
    if (R, N, K) != (M, weight.N, weight.K):
        raise ValueError("X must be [M, K] and Y [M, N]")
    _check(lib().qf_packed_matvec(ctypes.byref(weight), M, _ptr(X), ldx, _ptr(Y), ldy, f32,
                                  _stream()))
    return Y


def packed_matvec_grouped(weight: Packed, offsets, X, Y, rows=None, rows_div=1):
    """Y[r] = X[x(r)] W_e^T for r in offsets[e] .. offsets[e + 1] - 1; x(r) = r, or
    rows[r] // rows_div (a dispatch's slot_of and k)."""
    M, K, ldx = _mat(_bf16(X))
    R, N, ldy, f32 = _products(Y)
    if (N, K) != (weight.N, weight.K):
        raise ValueError("X must be [M, K] and Y [R, N]")
    _check(lib().qf_packed_matvec_grouped(ctypes.byref(weight),
                                          _typed(offsets, torch.int64, "offsets", (weight.E + 1,)),
                                          R, _typed(rows, torch.int32, "rows", (R,)), rows_div, M,
                                          _ptr(X), ldx, _ptr(Y), ldy, f32, _stream()))
    return Y


# -------------------------------------------- the 4-bit cache of keys and values, its attention
def _dense(t, dtype, name, shape=None):
    """As _typed, for a tensor that has to be there."""
    if t is None:
        raise ValueError(f"{name} is missing")
    return _typed(t, dtype, name, shape)


def kv_cache(fmt, k_codes, k_scales, v_codes, v_scales, k_S=None, v_S=None) -> KvCache:
    """Descriptor of a cache in pages: codes uint8 [pages, H, page, D/2], scales uint8 [pages, H, page, D/16]
    (nvfp4, with the heads' tensor scales k_S, v_S float32 [H]) or [pages, H, page, D/32] (mxfp4).  It holds
    references to the tensors, so their device memory stays allocated while the descriptor is alive."""
    block = {"nvfp4": 16, "mxfp4": 32}[fmt]
    if k_codes.dim() != 4:
        raise ValueError("codes must be [pages, H, page, D/2]")
    pages, H, page, half = k_codes.shape
    D = 2 * half
    codes, scales = (pages, H, page, half), (pages, H, page, D // block)
    if fmt == "nvfp4":
        S = _dense(k_S, torch.float32, "k_S", (H,)), _dense(v_S, torch.float32, "v_S", (H,))
    else:
        S = None, None
    c = KvCache(pages, page, H, D, FMT[fmt], _dense(k_codes, torch.uint8, "k_codes", codes),
                _dense(k_scales, torch.uint8, "k_scales", scales),
                _dense(v_codes, torch.uint8, "v_codes", codes),
                _dense(v_scales, torch.uint8, "v_scales", scales), *S)
    c._tensors = (k_codes, k_scales, v_codes, v_scales, k_S, v_S)
    return c


def kv_sequences(lens, table, offsets=None, max_len=None) -> KvSeqs:
    """Descriptor of the sequences of a call: lens int32 [B] tokens of each, the call's included; table int32
    [B, cols] their pages; offsets int64 [B+1] their rows of the call (None: one each); max_len a bound on lens
    (None: what the table's rows hold, known when a cache is).  Holds references to the tensors, whose values
    may change between calls."""
    B, cols = table.shape
    if max_len is not None and max_len < 0:
        raise ValueError("max_len is negative")
    q = KvSeqs(B, _typed(offsets, torch.int64, "offsets", (B + 1,)), _dense(lens, torch.int32, "lens", (B,)),
               _dense(table, torch.int32, "table"), cols, -1 if max_len is None else max_len)
    q._tensors = (offsets, lens, table)
    return q


def _bounded(cache, seqs):
    """seqs with max_len filled in."""
    if seqs.max_len >= 0:
        return seqs
    return KvSeqs(seqs.B, seqs.offsets, seqs.lens, seqs.table, seqs.cols, min(seqs.cols * cache.page, (1 << 30) - 1))


def _heads(x, name, width=None):
    R, C, ld = _mat(_bf16(x))
    if width is not None and C != width:
        raise ValueError(f"{name} must have {width} columns")
    return R, C, ld


def kv_write(cache: KvCache, seqs: KvSeqs, K, V):
    """Quantizes the new tokens' K, V [T, H D] into their sequences' pages."""
    T, C, ldk = _heads(K, "K", cache.H * cache.D)
    T2, _, ldv = _heads(V, "V", C)
    if T2 != T:
        raise ValueError("K and V must have a row for every token")
    _check(lib().qf_kv_write(ctypes.byref(cache), ctypes.byref(_bounded(cache, seqs)), T, _ptr(K), ldk, _ptr(V), ldv,
                             _stream()))


def kv_read(cache: KvCache, seqs: KvSeqs, K=None, V=None):
    """The tokens' K, V [T, H D] (either may be None) as the cache holds them."""
    T, ld = None, [0, 0]
    for i, (x, name) in enumerate(((K, "K"), (V, "V"))):
        if x is not None:
            R, _, ld[i] = _heads(x, name, cache.H * cache.D)
            if T not in (None, R):
                raise ValueError("K and V must have a row for every token")
            T = R
    if T is None:
        return K, V
    _check(lib().qf_kv_read(ctypes.byref(cache), ctypes.byref(_bounded(cache, seqs)), T, _ptr(K), ld[0], _ptr(V), ld[1],
                            _stream()))
    return K, V


def kv_attention_workspace(cache: KvCache, seqs: KvSeqs, T, Hq, window=0, device="cuda"):
    n = ctypes.c_size_t()
    _check(lib().qf_kv_attention_workspace_size(ctypes.byref(cache), ctypes.byref(_bounded(cache, seqs)), T, Hq, window,
                                                ctypes.byref(n)))
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def kv_attention(cache: KvCache, seqs: KvSeqs, Q, O, ws, scale=None, window=0, lse=None):
    """Causal attention of Q [T, Hq D] over the cached tokens into O [T, Hq D] and lse float32 [T, Hq]; scale
    None: 1 / sqrt D; window > 0: only the last `window` positions up to a token's own."""
    T, C, ldq = _heads(Q, "Q")
    T2, _, ldo = _heads(O, "O", C)
    if T2 != T:
        raise ValueError("O must have the shape of Q")
    if C % cache.D:
        raise ValueError("Q must be [T, Hq D]")
    Hq = C // cache.D
    _check(lib().qf_kv_attention(ctypes.byref(cache), ctypes.byref(_bounded(cache, seqs)), T, _ptr(Q), ldq, Hq,
                                 cache.D ** -0.5 if scale is None else float(scale), window, _ptr(O), ldo,
                                 _typed(lse, torch.float32, "lse", (T, Hq)), _ptr(ws), ws.numel() * ws.element_size(),
                                 _stream()))
    return O


# ------------------------------------------------- adapters of many requests, not merged
def adapters(A, B, scale, ranks=None) -> Adapters:
    """Descriptor of n adapters beside one weight [N, K]: A bf16 [n, r, K], B bf16 [n, N, r], scale float32 [n],
    ranks int32 [n] (None: all r).  Holds references to the tensors."""
    n, r, K = A.shape
    N = B.shape[1]
    a = Adapters(n, r, N, K, _dense(_bf16(A), A.dtype, "A"), _dense(_bf16(B), B.dtype, "B", (n, N, r)),
                 _dense(scale, torch.float32, "scale", (n,)), _typed(ranks, torch.int32, "ranks", (n,)))
    a._tensors = (A, B, scale, ranks)
    return a


def lora_rows_workspace(a: Adapters, M, device="cuda"):
    n = ctypes.c_size_t()
    _check(lib().qf_lora_rows_workspace_size(ctypes.byref(a), M, ctypes.byref(n)))
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def lora_rows(a: Adapters, ids, X, Y, ws, base=None):
    """Y [M, N] (bf16 or float32) = base + scale[a] (X A_a^T) B_a^T with a = ids[m] (int32 [M], outside 0 .. n - 1:
    none).  base: of Y's type, may be Y itself; None: zeros."""
    M, K, ldx = _mat(_bf16(X))
    R, N, ldy, f32 = _products(Y)
    if (R, N, K) != (M, a.N, a.K):
        raise ValueError("X must be [M, K] and Y [M, N]")
    ldb = 0
    if base is not None:
        R2, N2, ldb, f2 = _products(base)
        if (R2, N2, f2) != (R, N, f32):
            raise ValueError("base must have the shape and type of Y")
    _check(lib().qf_lora_rows(ctypes.byref(a), _dense(ids, torch.int32, "ids", (M,)), M, _ptr(X), ldx, _ptr(base), ldb,
                              _ptr(Y), ldy, f32, _ptr(ws), ws.numel() * ws.element_size(), _stream()))
    return Y


# ------------------------------------------------------------------ QAD distillation loss
def qad_kl(zt, zs, row_kl, loss=None, grad=None, agree=None, grad_scale=None):
    """Forward KL of Eq. qad-objective per token (row_kl), its mean (loss), the student-logit
    gradient grad_scale * (p_S - p_T) (default grad_scale = 1/L) and top-1 agreement."""
    L, V, ldt = _rows(_bf16(zt))
    L2, V2, lds = _rows(_bf16(zs))
    if (L2, V2) != (L, V):
        raise ValueError("teacher and student logits must have the same shape")
    ldg = 0
    if grad is not None:
        _, _, ldg = _rows(_bf16(grad))
    gs = (1.0 / L if L else 1.0) if grad_scale is None else float(grad_scale)
    _check(lib().qf_qad_kl(_ptr(zt), ldt, _ptr(zs), lds, L, V, gs, _ptr(row_kl), _ptr(loss),
                           _ptr(grad), ldg, _ptr(agree), _stream()))


# --------------------------------------------------------------- engine-native export / sync
def export_fused(members, fmt, codes, scales, w_amax=None, weight_scale_2=None, a_amax=None,
                 input_scale=None):
    """Fused-projection export: members are bf16 [rows_i, K] tensors (row-contiguous)."""
    K = members[0].shape[1]
    arr = (Member * len(members))()
    for i, m in enumerate(members):
        R, Km, ld = _rows(_bf16(m))
        if Km != K:
            raise ValueError("members must share K")
        arr[i] = Member(_ptr(m), R, ld)
    _check(lib().qf_export_fused(FMT[fmt], arr, len(members), K, _ptr(codes), _ptr(scales),
                                 _ptr(w_amax), _ptr(weight_scale_2), _ptr(a_amax),
                                 _ptr(input_scale), _stream()))


def payload_layout(fmt, N, K) -> PayloadLayout:
    L = PayloadLayout()
    _check(lib().qf_payload_layout_of(FMT[fmt], N, K, ctypes.byref(L)))
    return L


def payload_write_header(fmt, N, K, payload):
    _check(lib().qf_payload_write_header(FMT[fmt], N, K, _ptr(payload), _stream()))

"""Python binding of libscalify.so (include/scalify.h): argument marshalling only.

Every step of the scaled matmul, rescale and cast runs in the HIP kernels of
the library; this module turns torch device tensors into the C structs, picks
the current HIP stream, allocates workspaces with torch and raises on a
non-OK status. There is no fallback: if the library is missing, importing it
raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import torch

E4M3, E5M2, F16, F32 = 0, 1, 2, 3
RESCALE_NONE, RESCALE_AMAX, RESCALE_DELAYED = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_GELU_TANH, ACT_SILU = 0, 1, 2, 3

STATUS_NAMES = {0: "SCALIFY_OK", 1: "SCALIFY_ERR_NULL", 2: "SCALIFY_ERR_DTYPE",
                3: "SCALIFY_ERR_SHAPE", 4: "SCALIFY_ERR_LAYOUT", 5: "SCALIFY_ERR_ALIGN",
                6: "SCALIFY_ERR_WORKSPACE", 7: "SCALIFY_ERR_VALUE", 8: "SCALIFY_ERR_HIP"}

# storage element type of each format (codes are carried as raw bits)
STORAGE_DTYPE = {E4M3: torch.uint8, E5M2: torch.uint8, F16: torch.int16, F32: torch.float32}

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libscalify.so")


class ScalifyError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} "
                         f"({string_of(status)})")


class CScaledArray(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("trans", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld", ctypes.c_int64)]


class CMatmulOpts(ctypes.Structure):
    _fields_ = [("out_dtype", ctypes.c_int32), ("rescale", ctypes.c_int32),
                ("target_log2", ctypes.c_int32), ("saturate", ctypes.c_int32),
                ("acc_out", ctypes.c_void_p), ("amax_out", ctypes.c_void_p),
                ("events", ctypes.c_void_p), ("amax_in", ctypes.c_void_p),
                ("residual", ctypes.POINTER(CScaledArray)), ("activation", ctypes.c_int32),
                ("pre_out", ctypes.c_void_p), ("a_channel_scale", ctypes.c_void_p),
                ("b_channel_scale", ctypes.c_void_p), ("a_block_scale", ctypes.c_void_p),
                ("b_block_scale", ctypes.c_void_p)]


class CAttentionOpts(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("batch", ctypes.c_int64), ("softmax_scale", ctypes.c_float),
                ("q_start", ctypes.c_void_p), ("k_start", ctypes.c_void_p), ("k_len", ctypes.c_void_p),
                ("max_q", ctypes.c_int64), ("max_k", ctypes.c_int64)]


EXPORTED = ("scalify_matmul_scale_log2", "scalify_matmul_workspace_size",
            "scalify_matmul_workspace_size_opts", "scalify_matmul",
            "scalify_rescale_workspace_size", "scalify_rescale", "scalify_cast",
            "scalify_set_scaling", "scalify_status_string", "scalify_layernorm_fwd",
            "scalify_layernorm_bwd_workspace_size", "scalify_layernorm_bwd",
            "scalify_mx_packed_bytes", "scalify_mx_pack_block_scales",
            "scalify_matmul_noalloc", "scalify_rmsnorm_fwd",
            "scalify_rmsnorm_bwd_workspace_size", "scalify_rmsnorm_bwd",
            "scalify_attention_fwd_workspace_size", "scalify_attention_fwd",
            "scalify_attention_bwd_workspace_size", "scalify_attention_bwd",
            "scalify_cross_entropy_fwd_workspace_size", "scalify_cross_entropy_fwd",
            "scalify_cross_entropy_bwd_workspace_size", "scalify_cross_entropy_bwd",
            "scalify_distillation_fwd_workspace_size", "scalify_distillation_fwd",
            "scalify_distillation_bwd_workspace_size", "scalify_distillation_bwd")

_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libscalify.so (built by paper_2407_17353_amd/build.py). Raises
    FileNotFoundError when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: run paper_2407_17353_amd/build.py")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.scalify_matmul_scale_log2.argtypes = [i64]
    lib.scalify_matmul_scale_log2.restype = i32
    lib.scalify_mx_packed_bytes.argtypes = [i64, i64]
    lib.scalify_mx_packed_bytes.restype = i64
    lib.scalify_mx_pack_block_scales.argtypes = [vp, i64, i64, i64, vp, vp]
    lib.scalify_mx_pack_block_scales.restype = ctypes.c_int
    lib.scalify_matmul_workspace_size.argtypes = [i64, i64, i32, i32]
    lib.scalify_matmul_workspace_size.restype = ctypes.c_size_t
    lib.scalify_matmul_workspace_size_opts.argtypes = [i64, i64, P(CMatmulOpts)]
    lib.scalify_matmul_workspace_size_opts.restype = ctypes.c_size_t
    lib.scalify_matmul.argtypes = [P(CScaledArray), P(CScaledArray), P(CScaledArray),
                                   P(CMatmulOpts), vp, ctypes.c_size_t, vp]
    lib.scalify_matmul.restype = ctypes.c_int
    lib.scalify_matmul_noalloc.argtypes = [P(CScaledArray), P(CScaledArray), P(CScaledArray),
                                           P(CMatmulOpts), vp]
    lib.scalify_matmul_noalloc.restype = ctypes.c_int
    lib.scalify_rescale_workspace_size.argtypes = [i64]
    lib.scalify_rescale_workspace_size.restype = ctypes.c_size_t
    lib.scalify_rescale.argtypes = [P(CScaledArray), P(CScaledArray), i32, i32, i32, vp,
                                    ctypes.c_size_t, vp]
    lib.scalify_rescale.restype = ctypes.c_int
    lib.scalify_cast.argtypes = [P(CScaledArray), P(CScaledArray), i32, vp]
    lib.scalify_cast.restype = ctypes.c_int
    lib.scalify_set_scaling.argtypes = [P(CScaledArray), P(CScaledArray), i32, i32, vp]
    lib.scalify_set_scaling.restype = ctypes.c_int
    f32 = ctypes.c_float
    lib.scalify_layernorm_fwd.argtypes = [P(CScaledArray), vp, vp, f32, P(CScaledArray), i32, vp, vp]
    lib.scalify_layernorm_fwd.restype = ctypes.c_int
    lib.scalify_layernorm_bwd_workspace_size.argtypes = [i64, i64]
    lib.scalify_layernorm_bwd_workspace_size.restype = ctypes.c_size_t
    lib.scalify_layernorm_bwd.argtypes = [P(CScaledArray), P(CScaledArray), vp, f32, P(CScaledArray),
                                          vp, vp, i32, i32, i32, vp, vp, vp, ctypes.c_size_t, vp]
    lib.scalify_layernorm_bwd.restype = ctypes.c_int
    lib.scalify_rmsnorm_fwd.argtypes = [P(CScaledArray), P(CScaledArray), vp, f32, P(CScaledArray),
                                        P(CScaledArray), vp, vp, i32, i32, vp, vp]
    lib.scalify_rmsnorm_fwd.restype = ctypes.c_int
    lib.scalify_rmsnorm_bwd_workspace_size.argtypes = [i64, i64]
    lib.scalify_rmsnorm_bwd_workspace_size.restype = ctypes.c_size_t
    lib.scalify_rmsnorm_bwd.argtypes = [P(CScaledArray), P(CScaledArray), P(CScaledArray), vp, f32,
                                        P(CScaledArray), vp, i32, i32, i32, vp, vp, vp,
                                        ctypes.c_size_t, vp]
    lib.scalify_rmsnorm_bwd.restype = ctypes.c_int
    A = P(CScaledArray)
    lib.scalify_attention_fwd_workspace_size.argtypes = [i64, i64, P(CAttentionOpts)]
    lib.scalify_attention_fwd_workspace_size.restype = ctypes.c_size_t
    lib.scalify_attention_fwd.argtypes = [A, A, A, A, vp, P(CAttentionOpts), i32, vp, ctypes.c_size_t, vp]
    lib.scalify_attention_fwd.restype = ctypes.c_int
    lib.scalify_attention_bwd_workspace_size.argtypes = [i64, i64, P(CAttentionOpts), i32]
    lib.scalify_attention_bwd_workspace_size.restype = ctypes.c_size_t
    lib.scalify_attention_bwd.argtypes = [A, A, A, A, A, vp, A, A, A, P(CAttentionOpts), i32, i32, i32, vp,
                                          vp, ctypes.c_size_t, vp]
    lib.scalify_attention_bwd.restype = ctypes.c_int
    sz = ctypes.c_size_t
    lib.scalify_cross_entropy_fwd_workspace_size.argtypes = [i64, i64, i64, i32]
    lib.scalify_cross_entropy_fwd_workspace_size.restype = sz
    lib.scalify_cross_entropy_fwd.argtypes = [A, A, vp, vp, vp, vp, vp, sz, vp]
    lib.scalify_cross_entropy_fwd.restype = ctypes.c_int
    lib.scalify_cross_entropy_bwd_workspace_size.argtypes = [i64, i64, i64, i32, i32]
    lib.scalify_cross_entropy_bwd_workspace_size.restype = sz
    lib.scalify_cross_entropy_bwd.argtypes = [vp, vp, A, A, vp, vp, vp, A, A, i32, i32, i32, vp, vp, sz, vp]
    lib.scalify_cross_entropy_bwd.restype = ctypes.c_int
    lib.scalify_distillation_fwd_workspace_size.argtypes = [i64, i64, i64, i64, i32]
    lib.scalify_distillation_fwd_workspace_size.restype = sz
    lib.scalify_distillation_fwd.argtypes = [A, A, A, vp, f32, vp, vp, vp, vp, vp, sz, vp]
    lib.scalify_distillation_fwd.restype = ctypes.c_int
    lib.scalify_distillation_bwd_workspace_size.argtypes = [i64, i64, i64, i64, i32, i32]
    lib.scalify_distillation_bwd_workspace_size.restype = sz
    lib.scalify_distillation_bwd.argtypes = [vp, vp, A, A, A, vp, f32, vp, vp, vp, A, A, i32, i32, i32, vp, vp, sz, vp]
    lib.scalify_distillation_bwd.restype = ctypes.c_int
    lib.scalify_status_string.argtypes = [i32]
    lib.scalify_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


def string_of(status: int) -> str:
    return load_library().scalify_status_string(int(status)).decode()


@dataclass
class ScaledArray:
    """A ScaledArray (data, scale) with value = decode(data) * scale
    (Section 2 of the paper). `data` is the STORED matrix as a 2-D tensor
    whose rows are contiguous (stride(1) == 1; stride(0) is the leading
    dimension); with trans=True it stores the transpose of the logical
    matrix. `scale` is a one-element float32 device tensor or None (scale 1)."""
    data: torch.Tensor
    fmt: int
    scale: Optional[torch.Tensor] = None
    trans: bool = False

    @property
    def shape(self):
        r, c = self.data.shape
        return (c, r) if self.trans else (r, c)

    def c_struct(self) -> CScaledArray:
        d = self.data
        if d.dim() != 2:
            raise ValueError("ScaledArray data must be 2-D")
        rows, cols = d.shape
        ptr, ld = None, 0
        if rows * cols:
            ld, one = d.stride()
            if one != 1:
                raise ValueError("ScaledArray rows must be contiguous")
            ptr = d.data_ptr()
        if self.trans:
            rows, cols = cols, rows
        return CScaledArray(ptr, self.scale.data_ptr() if self.scale is not None else None,
                            int(self.fmt), int(bool(self.trans)), rows, cols, ld)


def _stream_handle(stream) -> Optional[int]:
    if stream is None:  # (the handle alone: a torch.cuda.Stream object takes 2.4 us more)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _check(status: int, where: str):
    if status != 0:
        raise ScalifyError(status, where)


def scalify_matmul_scale_log2(K: int) -> int:
    return int(load_library().scalify_matmul_scale_log2(int(K)))


def scalify_mx_packed_bytes(rows: int, K: int) -> int:
    """Bytes of the packed form of an MX block-scale array (rows x K)."""
    return int(load_library().scalify_mx_packed_bytes(int(rows), int(K)))


def scalify_mx_pack_block_scales(src: torch.Tensor, K: int, stream=None) -> torch.Tensor:
    """Pack row-major E8M0 block-scale bytes src [rows, ld] (uint8 device
    tensor, ld >= ceil(K / 32), byte [r, k // 32] scaling row r's k) into the
    order scalify_matmul reads; returns a new uint8 device tensor."""
    if src.dtype != torch.uint8 or src.dim() != 2 or src.stride(1) != 1:
        raise ValueError("src: uint8 [rows, ld] with unit column stride")
    rows = src.shape[0]
    dst = torch.empty(max(scalify_mx_packed_bytes(rows, K), 4), dtype=torch.uint8,
                      device=src.device)
    st = load_library().scalify_mx_pack_block_scales(
        src.data_ptr() if src.numel() else None, rows, int(K), src.stride(0), dst.data_ptr(),
        _stream_handle(stream))
    _check(st, "scalify_mx_pack_block_scales")
    return dst[:scalify_mx_packed_bytes(rows, K)]


def scalify_matmul_workspace_size(M: int, N: int, out_fmt: int, rescale: int = RESCALE_AMAX) -> int:
    return int(load_library().scalify_matmul_workspace_size(M, N, out_fmt, rescale))


def scalify_matmul_workspace_size_opts(M: int, N: int, out_fmt: int, rescale: int = RESCALE_AMAX,
                                       fused: bool = False) -> int:
    """Workspace bytes of a call with (fused=True) or without a fused
    residual add, activation or pre_out export."""
    opts = CMatmulOpts(int(out_fmt), int(rescale), 0, 1, None, None, None, None, None,
                       ACT_RELU if fused else ACT_NONE, None)
    return int(load_library().scalify_matmul_workspace_size_opts(M, N, ctypes.byref(opts)))


def scalify_rescale_workspace_size(n: int) -> int:
    return int(load_library().scalify_rescale_workspace_size(n))


def workspace(nbytes: int, device) -> torch.Tensor:
    """Device workspace of nbytes, 256-byte aligned (torch allocations are)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def scalify_matmul(a: ScaledArray, b: ScaledArray, out: ScaledArray, *, rescale: int = RESCALE_AMAX,
                   target_log2: int = 0, saturate: bool = True, acc_out: torch.Tensor = None,
                   amax_out: torch.Tensor = None, amax_in: torch.Tensor = None,
                   residual: "ScaledArray" = None, activation: int = ACT_NONE,
                   pre_out: torch.Tensor = None, a_channel_scale: torch.Tensor = None,
                   b_channel_scale: torch.Tensor = None, a_block_scale: torch.Tensor = None,
                   b_block_scale: torch.Tensor = None,
                   ws: torch.Tensor = None, stream=None, events=None) -> None:
    """Scaled matmul (Section 3.2) with the fused dynamic or delayed rescale
    and cast (Section 3.3); see scalify_matmul in include/scalify.h.
    `amax_in` (RESCALE_DELAYED): one-element fp32 device tensor holding the
    statistic of an earlier call (its `amax_out`; may be the same tensor).
    `residual`: ScaledArray [M, N] added by the scaled add rule before the
    `activation` (ACT_*); a row broadcast as `bias.expand(M, N)` (stride 0)
    adds one row to every row. `pre_out`: fp32 [M, N] device tensor that
    receives the pre-cast value w (validation). `a_channel_scale` /
    `b_channel_scale`: contiguous fp32 device tensors [M] / [N] of powers of
    two, channel scales of a's rows / b's columns. `a_block_scale` /
    `b_block_scale`: MX block scales (E8M0, one per 32 k) of a's rows / b's
    columns, as returned by scalify_mx_pack_block_scales (uint8 device
    tensors of scalify_mx_packed_bytes(M or N, K) bytes).
    `events`: an optional sequence of 3 torch.cuda.Event(enable_timing=True)
    recorded before the GEMM kernel, after it and after the epilogue (None
    entries are skipped)."""
    lib = load_library()
    M, _ = a.shape
    _, N = b.shape
    opts, keep = _matmul_opts(a, out, rescale, target_log2, saturate, acc_out, amax_out, amax_in,
                              residual, activation, pre_out, a_channel_scale, b_channel_scale,
                              a_block_scale, b_block_scale, stream, events)
    if ws is None:
        ws = workspace(lib.scalify_matmul_workspace_size_opts(M, N, ctypes.byref(opts)),
                       a.data.device)
    ca, cb, co = a.c_struct(), b.c_struct(), out.c_struct()
    st = lib.scalify_matmul(ctypes.byref(ca), ctypes.byref(cb), ctypes.byref(co), ctypes.byref(opts),
                            ws.data_ptr(), ws.numel(), _stream_handle(stream))
    _check(st, "scalify_matmul")


def scalify_matmul_noalloc(a: ScaledArray, b: ScaledArray, out: ScaledArray, *,
                           rescale: int = RESCALE_AMAX, target_log2: int = 0,
                           saturate: bool = True, acc_out: torch.Tensor = None,
                           amax_out: torch.Tensor = None, amax_in: torch.Tensor = None,
                           residual: "ScaledArray" = None, activation: int = ACT_NONE,
                           pre_out: torch.Tensor = None, a_channel_scale: torch.Tensor = None,
                           b_channel_scale: torch.Tensor = None,
                           a_block_scale: torch.Tensor = None, b_block_scale: torch.Tensor = None,
                           stream=None, events=None) -> None:
    """scalify_matmul with the library's static workspace (no allocation by
    the library or by this binding); see scalify_matmul_noalloc in
    include/scalify.h for its size limit and its sharing rules."""
    lib = load_library()
    opts, keep = _matmul_opts(a, out, rescale, target_log2, saturate, acc_out, amax_out, amax_in,
                              residual, activation, pre_out, a_channel_scale, b_channel_scale,
                              a_block_scale, b_block_scale, stream, events)
    ca, cb, co = a.c_struct(), b.c_struct(), out.c_struct()
    st = lib.scalify_matmul_noalloc(ctypes.byref(ca), ctypes.byref(cb), ctypes.byref(co),
                                    ctypes.byref(opts), _stream_handle(stream))
    _check(st, "scalify_matmul_noalloc")


def _matmul_opts(a, out, rescale, target_log2, saturate, acc_out, amax_out, amax_in, residual,
                 activation, pre_out, a_channel_scale, b_channel_scale, a_block_scale,
                 b_block_scale, stream, events):
    """The scalify_matmul_opts struct of a call, and the ctypes objects it
    points to (kept alive by the caller until the call returns)."""
    M, K = a.shape
    N = out.shape[1]
    ev_arr = None
    if events is not None:
        for e in events:
            if e is not None and not e.cuda_event:       # torch creates its events lazily, on first record
                e.record(stream if stream is not None else torch.cuda.current_stream())
        ev_arr = (ctypes.c_void_p * 3)(*[e.cuda_event if e is not None else None for e in events])
    opts = CMatmulOpts(int(out.fmt), int(rescale), int(target_log2), int(bool(saturate)),
                       acc_out.data_ptr() if acc_out is not None else None,
                       amax_out.data_ptr() if amax_out is not None else None,
                       ctypes.cast(ev_arr, ctypes.c_void_p) if ev_arr is not None else None,
                       amax_in.data_ptr() if amax_in is not None else None,
                       None, int(activation), pre_out.data_ptr() if pre_out is not None else None,
                       a_channel_scale.data_ptr() if a_channel_scale is not None else None,
                       b_channel_scale.data_ptr() if b_channel_scale is not None else None,
                       a_block_scale.data_ptr() if a_block_scale is not None else None,
                       b_block_scale.data_ptr() if b_block_scale is not None else None)
    for t, rows in ((a_block_scale, M), (b_block_scale, N)):
        if t is not None and (t.dtype != torch.uint8 or not t.is_contiguous() or
                              t.numel() != scalify_mx_packed_bytes(rows, K)):
            raise ValueError("block scales: packed by scalify_mx_pack_block_scales")
    cr = residual.c_struct() if residual is not None else None
    if cr is not None:
        opts.residual = ctypes.pointer(cr)
    return opts, (ev_arr, cr)


def scalify_rescale(x: ScaledArray, out: ScaledArray, *, mode: int = RESCALE_AMAX, target_log2: int = 0,
                    saturate: bool = True, ws: torch.Tensor = None, stream=None) -> None:
    """Dynamic rescale (Section 3.3): amax -> power of two -> rebalance, plus cast."""
    lib = load_library()
    if ws is None:
        ws = workspace(scalify_rescale_workspace_size(x.data.numel()), x.data.device)
    ci, co = x.c_struct(), out.c_struct()
    st = lib.scalify_rescale(ctypes.byref(ci), ctypes.byref(co), int(mode), int(target_log2),
                             int(bool(saturate)), ws.data_ptr(), ws.numel(), _stream_handle(stream))
    _check(st, "scalify_rescale")


def scalify_cast(x: ScaledArray, out: ScaledArray, *, saturate: bool = True, stream=None) -> None:
    """Cast of the data component; the scale is copied (Appendix A)."""
    ci, co = x.c_struct(), out.c_struct()
    st = load_library().scalify_cast(ctypes.byref(ci), ctypes.byref(co), int(bool(saturate)),
                                     _stream_handle(stream))
    _check(st, "scalify_cast")


def scalify_set_scaling(x: ScaledArray, out: ScaledArray, new_scale_log2: int, *, saturate: bool = True,
                        stream=None) -> None:
    """set_scaling (Section 3.1): output scale 2^new_scale_log2, data rebalanced."""
    ci, co = x.c_struct(), out.c_struct()
    st = load_library().scalify_set_scaling(ctypes.byref(ci), ctypes.byref(co), int(new_scale_log2),
                                            int(bool(saturate)), _stream_handle(stream))
    _check(st, "scalify_set_scaling")


# ----------------------------------------------------------------------------- helpers

def _ptr_or_none(t: Optional[torch.Tensor]):
    return t.data_ptr() if t is not None else None


def scalify_layernorm_fwd(x: ScaledArray, out: ScaledArray, *, gamma: torch.Tensor = None,
                          beta: torch.Tensor = None, eps: float = 1e-5, saturate: bool = True,
                          pre_out: torch.Tensor = None, stream=None) -> None:
    """Scaled LayerNorm forward (Appendix C.2): normalizes x's data, output
    scale 1; see scalify_layernorm_fwd in include/scalify.h. gamma, beta:
    fp32 [D] device tensors or None."""
    lib = load_library()
    cx, co = x.c_struct(), out.c_struct()
    st = lib.scalify_layernorm_fwd(ctypes.byref(cx), _ptr_or_none(gamma), _ptr_or_none(beta),
                                   float(eps), ctypes.byref(co), int(bool(saturate)),
                                   _ptr_or_none(pre_out), _stream_handle(stream))
    _check(st, "scalify_layernorm_fwd")


def scalify_layernorm_bwd_workspace_size(R: int, D: int) -> int:
    return int(load_library().scalify_layernorm_bwd_workspace_size(R, D))


def scalify_layernorm_bwd(dy: ScaledArray, x: ScaledArray, dx: ScaledArray, *,
                          gamma: torch.Tensor = None, eps: float = 1e-5,
                          rescale: int = RESCALE_AMAX, target_log2: int = 0,
                          saturate: bool = True, dgamma: torch.Tensor = None,
                          dbeta: torch.Tensor = None, amax_out: torch.Tensor = None,
                          pre_out: torch.Tensor = None, ws: torch.Tensor = None,
                          stream=None) -> None:
    """LayerNorm input gradient with its dynamic rescale (Section 4, Section
    3.3); see scalify_layernorm_bwd in include/scalify.h."""
    lib = load_library()
    R, D = x.shape
    if ws is None:
        ws = workspace(scalify_layernorm_bwd_workspace_size(R, D), x.data.device)
    cdy, cx, cdx = dy.c_struct(), x.c_struct(), dx.c_struct()
    st = lib.scalify_layernorm_bwd(ctypes.byref(cdy), ctypes.byref(cx), _ptr_or_none(gamma),
                                   float(eps), ctypes.byref(cdx), _ptr_or_none(dgamma),
                                   _ptr_or_none(dbeta), int(rescale), int(target_log2),
                                   int(bool(saturate)), _ptr_or_none(amax_out),
                                   _ptr_or_none(pre_out), ws.data_ptr(), ws.numel(),
                                   _stream_handle(stream))
    _check(st, "scalify_layernorm_bwd")


def _struct_or_none(x: Optional[ScaledArray]):
    return ctypes.byref(x.c_struct()) if x is not None else None


def _check_operands(arrays, tensors, vectors=(), stream=None):
    """The memory of a call: codes in their format's storage type, contiguous fp32
    tensors of their sizes (`vectors`: pairs of a tensor or None and its size), all on
    the device of the call's stream, whose address space the kernels run in."""
    dev = torch.cuda.current_device() if stream is None else stream.device_index
    where = [t.get_device() for t in tensors if t is not None]
    for x in arrays:
        if x is None:
            continue
        if x.data.dtype is not STORAGE_DTYPE[x.fmt]:
            raise ValueError(f"data: {STORAGE_DTYPE[x.fmt]} for format {x.fmt}")
        where.append(x.data.get_device())
        s = x.scale
        if s is not None:
            where.append(s.get_device())
            if s.dtype is not torch.float32 or s.numel() != 1:
                raise ValueError("scale: one fp32")
    for t, n in vectors:
        if t is not None:
            where.append(t.get_device())
            if t.dtype is not torch.float32 or t.numel() != n or not t.is_contiguous():
                raise ValueError(f"contiguous fp32 of {n} elements")
    if where.count(dev) != len(where):
        raise ValueError(f"every tensor: on cuda:{dev}, the call's device")


def scalify_rmsnorm_fwd(x: ScaledArray, out: ScaledArray, *, residual: ScaledArray = None,
                        sum_out: ScaledArray = None, gamma: torch.Tensor = None, eps: float = 1e-5,
                        row_scale: torch.Tensor = None, block_scale: torch.Tensor = None,
                        target_log2: int = 0, saturate: bool = True, pre_out: torch.Tensor = None,
                        stream=None) -> None:
    """Scaled RMS norm forward with the residual's scaled add; see
    scalify_rmsnorm_fwd in include/scalify.h. `sum_out` receives the sum (the
    residual stream), `row_scale` (contiguous fp32 [R]) or `block_scale` (uint8,
    scalify_mx_packed_bytes(R, D) bytes) the output's power-of-two scales, as
    scalify_matmul's a_channel_scale / a_block_scale take them."""
    R, D = x.shape
    if row_scale is not None and (row_scale.dtype != torch.float32 or not row_scale.is_contiguous() or
                                  row_scale.numel() != R):
        raise ValueError("row_scale: contiguous fp32 [R]")
    if block_scale is not None and (block_scale.dtype != torch.uint8 or not block_scale.is_contiguous() or
                                    block_scale.numel() != scalify_mx_packed_bytes(R, D)):
        raise ValueError("block_scale: contiguous uint8 [scalify_mx_packed_bytes(R, D)]")
    _check_operands((x, out, residual, sum_out), (block_scale, row_scale), ((gamma, D), (pre_out, R * D)), stream)
    st = load_library().scalify_rmsnorm_fwd(
        _struct_or_none(x), _struct_or_none(residual), _ptr_or_none(gamma), float(eps),
        _struct_or_none(sum_out), _struct_or_none(out), _ptr_or_none(row_scale),
        _ptr_or_none(block_scale), int(target_log2), int(bool(saturate)), _ptr_or_none(pre_out),
        _stream_handle(stream))
    _check(st, "scalify_rmsnorm_fwd")


def scalify_rmsnorm_bwd_workspace_size(R: int, D: int) -> int:
    return int(load_library().scalify_rmsnorm_bwd_workspace_size(R, D))


def scalify_rmsnorm_bwd(dy: ScaledArray, x: ScaledArray, dx: ScaledArray, *, dsum: ScaledArray = None,
                        gamma: torch.Tensor = None, eps: float = 1e-5, rescale: int = RESCALE_AMAX,
                        target_log2: int = 0, saturate: bool = True, dgamma: torch.Tensor = None,
                        amax_out: torch.Tensor = None, pre_out: torch.Tensor = None,
                        ws: torch.Tensor = None, stream=None) -> None:
    """RMS norm input gradient, plus the gradient `dsum` that reaches the
    normalized array itself, with its dynamic rescale; see scalify_rmsnorm_bwd
    in include/scalify.h."""
    lib = load_library()
    R, D = x.shape
    _check_operands((dy, x, dx, dsum), (ws,), ((gamma, D), (dgamma, D), (amax_out, 1), (pre_out, R * D)), stream)
    if ws is None:
        ws = _call_workspace(max(scalify_rmsnorm_bwd_workspace_size(R, D), 1), x.data.device, stream)
    st = lib.scalify_rmsnorm_bwd(
        _struct_or_none(dy), _struct_or_none(x), _struct_or_none(dsum), _ptr_or_none(gamma), float(eps),
        _struct_or_none(dx), _ptr_or_none(dgamma), int(rescale), int(target_log2), int(bool(saturate)),
        _ptr_or_none(amax_out), _ptr_or_none(pre_out), ws.data_ptr(), ws.numel(), _stream_handle(stream))
    _check(st, "scalify_rmsnorm_bwd")


def attention_opts(q: ScaledArray, heads: int, *, kv_heads: int = None, batch: int = 1, causal: bool = False,
                   softmax_scale: float = None, q_start: torch.Tensor = None, k_start: torch.Tensor = None,
                   k_len: torch.Tensor = None, max_q: int = 0, max_k: int = 0) -> CAttentionOpts:
    """scalify_attention_opts of a call (include/scalify.h). softmax_scale
    defaults to 1 / sqrt(head_dim); q_start, k_start ([batch + 1]) and k_len
    ([batch]) are contiguous int64 device tensors."""
    D = q.shape[1] // heads if heads > 0 and q.shape[1] % heads == 0 else 0
    for t, n in ((q_start, batch + 1), (k_start, batch + 1), (k_len, batch)):
        if t is not None and (t.dtype != torch.int64 or not t.is_contiguous() or t.numel() != n):
            raise ValueError("q_start, k_start: contiguous int64 [batch + 1]; k_len: [batch]")
    if softmax_scale is None:
        softmax_scale = D ** -0.5 if D else 1.0
    return CAttentionOpts(int(heads), int(heads if kv_heads is None else kv_heads), D, int(bool(causal)), int(batch),
                          float(softmax_scale), _ptr_or_none(q_start), _ptr_or_none(k_start), _ptr_or_none(k_len),
                          int(max_q), int(max_k))


def _seq_tensors(opts):
    return tuple(opts.get(k) for k in ("q_start", "k_start", "k_len"))


def _call_workspace(nbytes: int, device, stream) -> Optional[torch.Tensor]:
    """A workspace of the memory that belongs to `stream`, whose work on it is done
    before another allocation of that stream gets it."""
    if nbytes == 0:
        return None
    if stream is None:
        return workspace(nbytes, device)
    with torch.cuda.stream(stream):
        return workspace(nbytes, device)


def scalify_attention_fwd_workspace_size(rows_q: int, rows_k: int, opts: CAttentionOpts) -> int:
    return int(load_library().scalify_attention_fwd_workspace_size(rows_q, rows_k, ctypes.byref(opts)))


def scalify_attention_fwd(q: ScaledArray, k: ScaledArray, v: ScaledArray, out: ScaledArray, *, heads: int,
                          lse: torch.Tensor = None, saturate: bool = True, ws: torch.Tensor = None,
                          stream=None, **opts) -> None:
    """Attention forward; see scalify_attention_fwd in include/scalify.h. q and
    out: [rows, heads * head_dim], k and v: [rows, kv_heads * head_dim]; lse: an
    optional fp32 [heads, rows of q] device tensor. Further arguments: those of
    attention_opts."""
    lib = load_library()
    o = attention_opts(q, heads, **opts)
    _check_operands((q, k, v, out), (ws, *_seq_tensors(opts)), ((lse, q.shape[0] * heads),), stream)
    if ws is None:
        ws = _call_workspace(scalify_attention_fwd_workspace_size(q.shape[0], k.shape[0], o), q.data.device, stream)
    st = lib.scalify_attention_fwd(_struct_or_none(q), _struct_or_none(k), _struct_or_none(v), _struct_or_none(out),
                                   _ptr_or_none(lse), ctypes.byref(o), int(bool(saturate)), _ptr_or_none(ws),
                                   ws.numel() if ws is not None else 0, _stream_handle(stream))
    _check(st, "scalify_attention_fwd")


def scalify_attention_bwd_workspace_size(rows_q: int, rows_k: int, opts: CAttentionOpts,
                                         rescale: int = RESCALE_AMAX) -> int:
    return int(load_library().scalify_attention_bwd_workspace_size(rows_q, rows_k, ctypes.byref(opts), int(rescale)))


def scalify_attention_bwd(dout: ScaledArray, q: ScaledArray, k: ScaledArray, v: ScaledArray, out: ScaledArray,
                          lse: torch.Tensor, dq: ScaledArray, dk: ScaledArray, dv: ScaledArray, *, heads: int,
                          rescale: int = RESCALE_AMAX, target_log2: int = 0, saturate: bool = True,
                          amax_out: torch.Tensor = None, ws: torch.Tensor = None, stream=None, **opts) -> None:
    """Attention gradients with their rescales; see scalify_attention_bwd in
    include/scalify.h. out and lse: what the forward stored; amax_out: an
    optional fp32 [3] device tensor. Further arguments: those of attention_opts."""
    lib = load_library()
    o = attention_opts(q, heads, **opts)
    _check_operands((dout, q, k, v, out, dq, dk, dv), (ws, *_seq_tensors(opts)), ((lse, q.shape[0] * heads), (amax_out, 3)), stream)
    if ws is None:
        ws = _call_workspace(scalify_attention_bwd_workspace_size(q.shape[0], k.shape[0], o, rescale),
                             q.data.device, stream)
    st = lib.scalify_attention_bwd(_struct_or_none(dout), _struct_or_none(q), _struct_or_none(k), _struct_or_none(v),
                                   _struct_or_none(out), _ptr_or_none(lse), _struct_or_none(dq), _struct_or_none(dk),
                                   _struct_or_none(dv), ctypes.byref(o), int(rescale), int(target_log2),
                                   int(bool(saturate)), _ptr_or_none(amax_out), _ptr_or_none(ws),
                                   ws.numel() if ws is not None else 0, _stream_handle(stream))
    _check(st, "scalify_attention_bwd")


def _check_index(t: torch.Tensor, n: int, name: str):
    if t.dtype != torch.int64 or not t.is_contiguous() or t.numel() != n:
        raise ValueError(f"{name}: contiguous int64 of {n} elements")


def scalify_cross_entropy_fwd_workspace_size(R: int, V: int, D: int, w_fmt: int) -> int:
    return int(load_library().scalify_cross_entropy_fwd_workspace_size(R, V, D, int(w_fmt)))


def scalify_cross_entropy_fwd(x: ScaledArray, w: ScaledArray, labels: torch.Tensor, loss: torch.Tensor, *,
                              lse: torch.Tensor = None, row_scale: torch.Tensor = None, ws: torch.Tensor = None,
                              stream=None) -> None:
    """Softmax cross entropy of the rows of x (R x D) against the output matrix w
    (V x D); see scalify_cross_entropy_fwd in include/scalify.h. labels: contiguous
    int64 [R]; loss, lse and row_scale: contiguous fp32 [R], the last two optional."""
    R, D = x.shape
    V = w.shape[0]
    _check_index(labels, R, "labels")
    _check_operands((x, w), (labels, ws), ((loss, R), (lse, R), (row_scale, R)), stream)
    if ws is None:
        ws = _call_workspace(scalify_cross_entropy_fwd_workspace_size(R, V, D, w.fmt), x.data.device, stream)
    st = load_library().scalify_cross_entropy_fwd(
        _struct_or_none(x), _struct_or_none(w), labels.data_ptr(), _ptr_or_none(row_scale), loss.data_ptr(),
        _ptr_or_none(lse), _ptr_or_none(ws), ws.numel() if ws is not None else 0, _stream_handle(stream))
    _check(st, "scalify_cross_entropy_fwd")


def scalify_cross_entropy_bwd_workspace_size(R: int, V: int, D: int, w_fmt: int, rescale: int = RESCALE_AMAX) -> int:
    return int(load_library().scalify_cross_entropy_bwd_workspace_size(R, V, D, int(w_fmt), int(rescale)))


def scalify_cross_entropy_bwd(x: ScaledArray, w: ScaledArray, labels: torch.Tensor, lse: torch.Tensor, *,
                              dx: ScaledArray = None, dw: ScaledArray = None, dloss: torch.Tensor = None,
                              dloss_scale: torch.Tensor = None, row_scale: torch.Tensor = None,
                              rescale: int = RESCALE_AMAX, target_log2: int = 0, saturate: bool = True,
                              amax_out: torch.Tensor = None, ws: torch.Tensor = None, stream=None) -> None:
    """Gradients of the cross entropy with their rescales; see
    scalify_cross_entropy_bwd in include/scalify.h. lse: what the forward stored;
    dloss: contiguous fp32 [R] or None (1), times dloss_scale; amax_out: fp32 [2]."""
    R, D = x.shape
    V = w.shape[0]
    _check_index(labels, R, "labels")
    _check_operands((x, w, dx, dw), (labels, ws),
                    ((lse, R), (dloss, R), (dloss_scale, 1), (row_scale, R), (amax_out, 2)), stream)
    if ws is None:
        ws = _call_workspace(scalify_cross_entropy_bwd_workspace_size(R, V, D, w.fmt, rescale), x.data.device, stream)
    st = load_library().scalify_cross_entropy_bwd(
        _ptr_or_none(dloss), _ptr_or_none(dloss_scale), _struct_or_none(x), _struct_or_none(w), labels.data_ptr(),
        _ptr_or_none(row_scale), lse.data_ptr(), _struct_or_none(dx), _struct_or_none(dw), int(rescale),
        int(target_log2), int(bool(saturate)), _ptr_or_none(amax_out), _ptr_or_none(ws),
        ws.numel() if ws is not None else 0, _stream_handle(stream))
    _check(st, "scalify_cross_entropy_bwd")


def scalify_distillation_fwd_workspace_size(R: int, V: int, D: int, top: int, w_fmt: int) -> int:
    return int(load_library().scalify_distillation_fwd_workspace_size(R, V, D, top, int(w_fmt)))


def scalify_distillation_fwd(x: ScaledArray, w: ScaledArray, teacher: ScaledArray, index: torch.Tensor,
                             loss: torch.Tensor, *, temperature: float = 1.0, lse: torch.Tensor = None,
                             picked: torch.Tensor = None, row_scale: torch.Tensor = None, ws: torch.Tensor = None,
                             stream=None) -> None:
    """Distillation loss of the rows of x against a teacher's top logits; see
    scalify_distillation_fwd in include/scalify.h. teacher: [R, top]; index:
    contiguous int64 [R, top]; loss, lse: contiguous fp32 [R]; picked: fp32 [R, top]."""
    R, D = x.shape
    V, top = w.shape[0], teacher.shape[1]
    _check_index(index, R * top, "index")
    _check_operands((x, w, teacher), (index, ws), ((loss, R), (lse, R), (picked, R * top), (row_scale, R)), stream)
    if ws is None:
        ws = _call_workspace(scalify_distillation_fwd_workspace_size(R, V, D, top, w.fmt), x.data.device, stream)
    st = load_library().scalify_distillation_fwd(
        _struct_or_none(x), _struct_or_none(w), _struct_or_none(teacher), index.data_ptr(), float(temperature),
        _ptr_or_none(row_scale), loss.data_ptr(), _ptr_or_none(lse), _ptr_or_none(picked), _ptr_or_none(ws),
        ws.numel() if ws is not None else 0, _stream_handle(stream))
    _check(st, "scalify_distillation_fwd")


def scalify_distillation_bwd_workspace_size(R: int, V: int, D: int, top: int, w_fmt: int,
                                            rescale: int = RESCALE_AMAX) -> int:
    return int(load_library().scalify_distillation_bwd_workspace_size(R, V, D, top, int(w_fmt), int(rescale)))


def scalify_distillation_bwd(x: ScaledArray, w: ScaledArray, teacher: ScaledArray, index: torch.Tensor,
                             lse: torch.Tensor, picked: torch.Tensor, *, temperature: float = 1.0,
                             dx: ScaledArray = None, dw: ScaledArray = None, dloss: torch.Tensor = None,
                             dloss_scale: torch.Tensor = None, row_scale: torch.Tensor = None,
                             rescale: int = RESCALE_AMAX, target_log2: int = 0, saturate: bool = True,
                             amax_out: torch.Tensor = None, ws: torch.Tensor = None, stream=None) -> None:
    """Gradients of the distillation loss with their rescales; see
    scalify_distillation_bwd in include/scalify.h. lse, picked: what the forward stored."""
    R, D = x.shape
    V, top = w.shape[0], teacher.shape[1]
    _check_index(index, R * top, "index")
    _check_operands((x, w, teacher, dx, dw), (index, ws),
                    ((lse, R), (picked, R * top), (dloss, R), (dloss_scale, 1), (row_scale, R), (amax_out, 2)), stream)
    if ws is None:
        ws = _call_workspace(scalify_distillation_bwd_workspace_size(R, V, D, top, w.fmt, rescale), x.data.device,
                             stream)
    st = load_library().scalify_distillation_bwd(
        _ptr_or_none(dloss), _ptr_or_none(dloss_scale), _struct_or_none(x), _struct_or_none(w),
        _struct_or_none(teacher), index.data_ptr(), float(temperature), _ptr_or_none(row_scale), lse.data_ptr(),
        picked.data_ptr(), _struct_or_none(dx), _struct_or_none(dw), int(rescale), int(target_log2),
        int(bool(saturate)), _ptr_or_none(amax_out), _ptr_or_none(ws), ws.numel() if ws is not None else 0,
        _stream_handle(stream))
    _check(st, "scalify_distillation_bwd")


def empty_scaled(rows: int, cols: int, fmt: int, device, ld: int = None) -> ScaledArray:
    """Output ScaledArray [rows, cols] with leading dimension ld (default: cols
    rounded up to 16 elements) and a fresh scale tensor."""
    if ld is None:
        ld = max(16, (cols + 15) // 16 * 16)
    storage = torch.empty((rows, ld), dtype=STORAGE_DTYPE[fmt], device=device)
    return ScaledArray(storage[:, :cols], fmt, torch.empty(1, dtype=torch.float32, device=device))


def scale_tensor(log2: int, device) -> torch.Tensor:
    return torch.tensor([2.0 ** log2], dtype=torch.float32, device=device)

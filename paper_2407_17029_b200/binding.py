"""ctypes binding of the C-ABI library declared in ``include/qblora.h``.

Argument marshalling only: torch owns device memory and streams, every step of
the computation runs inside ``libqblora.so``.  Importing this module fails
loudly if the library has not been built (``python -m paper_2407_17029_b200.build``
or ``__graft_entry__.build()``); there is no fallback path.

Names follow the header: ``quantize_blockwise``, ``linear_fwd``, ``linear_bwd``,
``merge``, ``lowbit_gemm``.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass, field
from typing import List, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqblora.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT, ERR_TOO_LARGE = range(7)
FMT_CODEBOOK_ABSMAX, FMT_AFFINE_MINMAX = 0, 1
F32, BF16 = 0, 1
OP_QUANTIZE, OP_LINEAR_FWD, OP_LINEAR_BWD, OP_MERGE, OP_LOWBIT_GEMM, OP_MERGE_DENSE = range(6)
# qblora_scale_op: the parameter-free operator pair around the adapter (Sec. 3.2; Sec. 4 scale-operator ablation)
SCALE_AVGPOOL_REPEAT, SCALE_TRUNCATE_ZEROPAD, SCALE_SAMPLE_ZEROFILL = range(3)
# qblora_rope_layout, qblora_rope_scale
ROPE_HALF, ROPE_PAIRS = range(2)
ROPE_SCALE_NONE, ROPE_SCALE_LINEAR, ROPE_SCALE_BASE, ROPE_SCALE_BANDED = range(4)

EXPORTS = ["qblora_default_code_table", "qblora_workspace_bytes", "qblora_status_string",
           "qblora_device_status", "qblora_quantize_blockwise", "qblora_linear_fwd",
           "qblora_linear_bwd", "qablora_merge", "qablora_lowbit_gemm", "qblora_kernel_launches",
           "qblora_set_timing_events", "qablora_merge_noalloc", "qblora_merge_dense",
           "qblora_quantize_minmax_nbit", "qblora_debug_set_wait_limit", "qblora_debug_drop_load", "qblora_debug_hold_producer", "qblora_dense_gemm", "qblora_pack_codes", "qblora_unpack_codes",
           "qblora_rope_table", "qblora_rope", "qblora_rope_append", "qblora_kv_plan", "qblora_attention_workspace_bytes",
           "qblora_paged_attention"]


class _CQWeight(ctypes.Structure):
    _fields_ = [("d_in", ctypes.c_int32), ("d_out", ctypes.c_int32),
                ("block_in", ctypes.c_int32), ("block_out", ctypes.c_int32),
                ("qfmt", ctypes.c_int32), ("code", ctypes.c_float * 16),
                ("codes", ctypes.c_void_p), ("alpha", ctypes.c_void_p), ("beta", ctypes.c_void_p),
                ("code_bits", ctypes.c_int32)]


class _CAdapter(ctypes.Structure):
    _fields_ = [("lambda_in", ctypes.c_int32), ("lambda_out", ctypes.c_int32),
                ("rank", ctypes.c_int32), ("scaling", ctypes.c_float),
                ("A", ctypes.c_void_p), ("B", ctypes.c_void_p), ("scale_op", ctypes.c_int32)]


class _CHeads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class _CKVCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("page_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("n_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class _CRope(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("amplitude", ctypes.c_float), ("turns", ctypes.c_void_p)]


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build the CUDA library first "
                      "(python -m paper_2407_17029_b200.build); there is no CPU fallback")
_lib = ctypes.CDLL(LIB_PATH)
_lib.qblora_workspace_bytes.restype = ctypes.c_size_t
_lib.qblora_workspace_bytes.argtypes = [ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64]
_lib.qblora_status_string.restype = ctypes.c_char_p
_lib.qblora_status_string.argtypes = [ctypes.c_int]
_lib.qblora_default_code_table.argtypes = [ctypes.c_void_p]
_lib.qblora_device_status.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
_lib.qblora_quantize_blockwise.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int32, ctypes.c_int32,
                                           ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                           ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
_lib.qblora_quantize_minmax_nbit.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int32, ctypes.c_int32,
                                             ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                             ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
_lib.qblora_linear_fwd.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                   ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t,
                                   ctypes.c_void_p]
_lib.qblora_linear_bwd.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                   ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p,
                                   ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
_lib.qablora_merge.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                               ctypes.c_size_t, ctypes.c_void_p]
_lib.qablora_lowbit_gemm.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                     ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]


_lib.qablora_merge_noalloc.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
_lib.qblora_merge_dense.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                    ctypes.c_size_t, ctypes.c_void_p]
_lib.qblora_merge_dense.restype = ctypes.c_int
_lib.qblora_kernel_launches.restype = ctypes.c_uint64
_lib.qblora_kernel_launches.argtypes = []
_lib.qblora_set_timing_events.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
_lib.qblora_dense_gemm.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                   ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
_lib.qblora_pack_codes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                   ctypes.c_size_t, ctypes.c_void_p]
_lib.qblora_unpack_codes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
_lib.qblora_debug_set_wait_limit.argtypes = [ctypes.c_int64]
_lib.qblora_debug_drop_load.argtypes = [ctypes.c_int32]
_lib.qblora_debug_hold_producer.argtypes = [ctypes.c_int64]
_vp, _i32, _i64, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
_lib.qblora_rope_table.argtypes = [_i32, ctypes.c_double, _i32, ctypes.c_double, _i64, ctypes.c_double, ctypes.c_double, _vp]
_lib.qblora_rope.argtypes = [_vp, ctypes.c_int, _vp, _i64, _vp, _vp, _vp, _vp, _vp]
_lib.qblora_rope_append.argtypes = [_vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.qblora_kv_plan.argtypes = [_vp, _vp, _vp, _i32, _vp, _i32, _vp, _i32, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.qblora_attention_workspace_bytes.restype = _sz
_lib.qblora_attention_workspace_bytes.argtypes = [_vp, _i32, _i64]
_lib.qblora_paged_attention.argtypes = [_vp, _vp, _i32, _vp, _vp, _i32, _vp, _i64, ctypes.c_float, ctypes.c_int, _i32, _vp,
                                        _vp, _vp, _sz, _vp]


def kernel_launches() -> int:
    return int(_lib.qblora_kernel_launches())


def set_timing_events(start, stop) -> None:
    """Arm (torch.cuda.Event, already recorded once or created with enable_timing) or disarm (None, None)."""
    if start is None:
        _lib.qblora_set_timing_events(None, None)
    else:
        _lib.qblora_set_timing_events(start.cuda_event, stop.cuda_event)


def debug_set_wait_limit(cycles: int) -> None:
    """Test hook: device-side waits of kernels launched from now on give up after `cycles` cycles (0 = default)."""
    _check_plain(_lib.qblora_debug_set_wait_limit(int(cycles)))


def debug_drop_load(iteration: int) -> None:
    """Test hook: the next fused-contraction launch leaves out one weight load (see the header); negative = disarm."""
    _check_plain(_lib.qblora_debug_drop_load(int(iteration)))


def debug_hold_producer(cycles: int) -> None:
    """Test hook: the producers of the next adapted fused-contraction launch idle `cycles` cycles before their
    first adapter K-block (see the header); 0 = disarm."""
    _check_plain(_lib.qblora_debug_hold_producer(int(cycles)))


def _check_plain(status: int):
    if status != OK:
        raise RuntimeError(f"status {status}")


class QbloraError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {_lib.qblora_status_string(status).decode()} (status {status})")


def _check(status: int, where: str):
    if status != OK:
        raise QbloraError(status, where)


def status_string(status: int) -> str:
    return _lib.qblora_status_string(status).decode()


def default_code_table() -> List[float]:
    buf = (ctypes.c_float * 16)()
    _check(_lib.qblora_default_code_table(buf), "qblora_default_code_table")
    return list(buf)


@dataclass
class QWeight:
    """Frozen 4-bit weight: codes uint8 [d_out][d_in/2], alpha/beta fp32 [d_out/bo][d_in/bi] (device)."""
    d_out: int
    d_in: int
    block_in: int
    block_out: int
    qfmt: int
    code: List[float]
    codes: torch.Tensor
    alpha: torch.Tensor
    beta: Optional[torch.Tensor]
    code_bits: int = 4          # 4: codes one per nibble [d_out][d_in/2]; 2 / 3: dense storage [d_out][d_in*bits/8]

    def c_struct(self) -> _CQWeight:
        c = _CQWeight()
        c.d_in, c.d_out, c.block_in, c.block_out, c.qfmt = self.d_in, self.d_out, self.block_in, self.block_out, self.qfmt
        for j in range(16):
            c.code[j] = self.code[j] if self.code is not None else 0.0
        c.codes = self.codes.data_ptr()
        c.alpha = self.alpha.data_ptr()
        c.beta = self.beta.data_ptr() if self.beta is not None else None
        c.code_bits = int(self.code_bits)
        return c


@dataclass
class Adapter:
    """Balanced adapter: A bf16 [P][r], B bf16 [r][Q] (device); B None => A is the single matrix H [P][Q].
    scale_op picks the compress / restore operator pair (default: AvgPool & repeat_interleave)."""
    lambda_in: int
    lambda_out: int
    rank: int
    scaling: float
    A: torch.Tensor
    B: Optional[torch.Tensor]
    scale_op: int = SCALE_AVGPOOL_REPEAT

    def c_struct(self) -> _CAdapter:
        c = _CAdapter()
        c.lambda_in, c.lambda_out, c.rank, c.scaling = self.lambda_in, self.lambda_out, self.rank, self.scaling
        c.scale_op = int(self.scale_op)
        c.A = self.A.data_ptr()
        c.B = self.B.data_ptr() if self.B is not None else None
        return c


# the current stream's handle without building a Stream object, where this torch has that call (a microsecond a launch)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_ptr(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _raw_device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """A workspace or result of a call on `stream`, as one made under torch.cuda.stream(stream): memory of the current stream would
    be handed out again there as soon as a workspace is dropped, while the call's kernels on `stream` still use it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _dt(torch_dtype) -> int:
    if torch_dtype is torch.bfloat16:
        return BF16
    if torch_dtype is torch.float32:
        return F32
    raise ValueError(f"unsupported dtype {torch_dtype}")


def _ref(obj):
    return ctypes.byref(obj) if obj is not None else None


def workspace_bytes(op: int, qw: QWeight, ad: Optional[Adapter], tokens: int) -> int:
    cq = qw.c_struct()
    ca = ad.c_struct() if ad is not None else None
    return int(_lib.qblora_workspace_bytes(op, ctypes.byref(cq), _ref(ca), tokens))


def alloc_workspace(op: int, qw: QWeight, ad: Optional[Adapter], tokens: int, stream=None) -> torch.Tensor:
    n = max(workspace_bytes(op, qw, ad, tokens), 256)
    return _empty(n, torch.uint8, qw.codes.device, stream)


def device_status(ws: torch.Tensor, stream=None) -> int:
    return int(_lib.qblora_device_status(ws.data_ptr(), _stream_ptr(stream)))


def quantize_blockwise(W: torch.Tensor, block_in: int = 64, block_out: int = 1,
                       qfmt: int = FMT_CODEBOOK_ABSMAX, code: Optional[List[float]] = None,
                       stream=None, out: Optional[QWeight] = None) -> QWeight:
    """Quantizes W [d_out][d_in] (fp32 or bf16).  `out`: a QWeight of the same geometry whose tensors are
    overwritten (no allocation in the call)."""
    assert W.is_cuda and W.is_contiguous() and W.dim() == 2
    d_out, d_in = W.shape
    if qfmt == FMT_CODEBOOK_ABSMAX and code is None:
        code = default_code_table()
    if out is not None:
        assert (out.d_out, out.d_in, out.block_in, out.block_out, out.qfmt) == (d_out, d_in, block_in, block_out, qfmt)
        codes, alpha, beta = out.codes, out.alpha, out.beta
    else:
        codes = _empty((d_out, d_in // 2), torch.uint8, W.device, stream)
        alpha = _empty((max(d_out // block_out, 1), max(d_in // block_in, 1)), torch.float32, W.device, stream)
        beta = _empty(alpha.shape, torch.float32, W.device, stream) if qfmt == FMT_AFFINE_MINMAX else None
    ctab = (ctypes.c_float * 16)(*code) if code is not None else None
    st = _lib.qblora_quantize_blockwise(W.data_ptr(), _dt(W.dtype), d_out, d_in, block_in, block_out, qfmt,
                                        ctab, codes.data_ptr(), alpha.data_ptr(),
                                        beta.data_ptr() if beta is not None else None, _stream_ptr(stream))
    _check(st, "qblora_quantize_blockwise")
    return QWeight(d_out, d_in, block_in, block_out, qfmt, list(code) if code is not None else [0.0] * 16,
                   codes, alpha, beta)


def quantize_minmax_nbit(W: torch.Tensor, bits: int, block_in: int = 64, block_out: int = 1, stream=None) -> QWeight:
    """Min-max quantization of W [d_out][d_in] (fp32 or bf16) on a 2^bits-level grid (Eq. 1 with N = bits).
    The codes stay one per nibble, so the result is an ordinary min-max QWeight for every other call."""
    assert W.is_cuda and W.is_contiguous() and W.dim() == 2
    d_out, d_in = W.shape
    codes = _empty((d_out, d_in // 2), torch.uint8, W.device, stream)
    alpha = _empty((max(d_out // block_out, 1), max(d_in // block_in, 1)), torch.float32, W.device, stream)
    beta = _empty(alpha.shape, torch.float32, W.device, stream)
    st = _lib.qblora_quantize_minmax_nbit(W.data_ptr(), _dt(W.dtype), d_out, d_in, block_in, block_out, int(bits),
                                          codes.data_ptr(), alpha.data_ptr(), beta.data_ptr(), _stream_ptr(stream))
    _check(st, "qblora_quantize_minmax_nbit")
    return QWeight(d_out, d_in, block_in, block_out, FMT_AFFINE_MINMAX, [0.0] * 16, codes, alpha, beta)


def linear_fwd(qw: QWeight, ad: Optional[Adapter], X: torch.Tensor, out_dtype=torch.bfloat16,
               ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    assert X.is_cuda and X.is_contiguous() and X.dtype == torch.bfloat16
    T = X.shape[0]
    Y = out if out is not None else _empty((T, qw.d_out), out_dtype, X.device, stream)
    if ws is None:
        ws = alloc_workspace(OP_LINEAR_FWD, qw, ad, T, stream)
    cq = qw.c_struct()
    ca = ad.c_struct() if ad is not None else None
    st = _lib.qblora_linear_fwd(ctypes.byref(cq), _ref(ca), X.data_ptr(), T, Y.data_ptr(), _dt(Y.dtype),
                                ws.data_ptr(), ws.numel(), _stream_ptr(stream))
    _check(st, "qblora_linear_fwd")
    return Y


def linear_bwd(qw: QWeight, ad: Optional[Adapter], X: Optional[torch.Tensor], dY: torch.Tensor,
               dx_dtype=torch.bfloat16, need_dx: bool = True, need_da: bool = True, need_db: bool = True,
               ws: Optional[torch.Tensor] = None, outs: Optional[Tuple] = None, stream=None):
    """Returns (dX, dA, dB); entries are None where skipped."""
    assert dY.is_cuda and dY.is_contiguous() and dY.dtype == torch.bfloat16
    T = dY.shape[0]
    dev = dY.device
    if outs is not None:
        dX, dA, dB = outs
    else:
        dX = _empty((T, qw.d_in), dx_dtype, dev, stream) if need_dx else None
        dA = dB = None
        if ad is not None:
            if need_da:
                dA = _empty(tuple(ad.A.shape), torch.float32, dev, stream)
            if need_db and ad.B is not None:
                dB = _empty(tuple(ad.B.shape), torch.float32, dev, stream)
    if ws is None:
        ws = alloc_workspace(OP_LINEAR_BWD, qw, ad, T, stream)
    cq = qw.c_struct()
    ca = ad.c_struct() if ad is not None else None
    p = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    st = _lib.qblora_linear_bwd(ctypes.byref(cq), _ref(ca), p(X), dY.data_ptr(), T, p(dX),
                                _dt(dX.dtype) if dX is not None else BF16, p(dA), p(dB), ws.data_ptr(),
                                ws.numel(), _stream_ptr(stream))
    _check(st, "qblora_linear_bwd")
    return dX, dA, dB


def merge(qw: QWeight, ad: Adapter, in_place: bool = False, ws: Optional[torch.Tensor] = None,
          stream=None, beta_out: Optional[torch.Tensor] = None) -> QWeight:
    """QA-BLoRA merge: returns the weight with beta' (codes and alpha are shared, untouched).
    `beta_out`: preallocated fp32 tensor of beta's shape to receive beta'."""
    if qw.beta is None:
        raise QbloraError(ERR_INVALID_ARG, "qablora_merge")
    if beta_out is None:
        beta_out = qw.beta if in_place else _empty(qw.beta.shape, torch.float32, qw.beta.device, stream)
    if ws is None:
        ws = alloc_workspace(OP_MERGE, qw, ad, 0, stream)
    cq = qw.c_struct()
    ca = ad.c_struct()
    st = _lib.qablora_merge(ctypes.byref(cq), ctypes.byref(ca), beta_out.data_ptr(), ws.data_ptr(),
                            ws.numel(), _stream_ptr(stream))
    _check(st, "qablora_merge")
    return QWeight(qw.d_out, qw.d_in, qw.block_in, qw.block_out, qw.qfmt, qw.code, qw.codes, qw.alpha, beta_out, qw.code_bits)


def merge_dense(qw: QWeight, ad: Optional[Adapter], out: Optional[torch.Tensor] = None,
                ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Dense 16-bit merge: bf16 [d_out][d_in] = dequantized weight + s * dense adapter update."""
    W = out if out is not None else _empty((qw.d_out, qw.d_in), torch.bfloat16, qw.codes.device, stream)
    if ws is None:
        ws = alloc_workspace(OP_MERGE_DENSE, qw, ad, 0, stream)
    cq = qw.c_struct()
    ca = ad.c_struct() if ad is not None else None
    st = _lib.qblora_merge_dense(ctypes.byref(cq), _ref(ca), W.data_ptr(), ws.data_ptr(), ws.numel(),
                                 _stream_ptr(stream))
    _check(st, "qblora_merge_dense")
    return W


def merge_noalloc(qw: QWeight, ad: Adapter, beta_out: torch.Tensor, stream=None) -> QWeight:
    """qablora_merge_noalloc: merge into the caller's ``beta_out`` using the library's built-in scratch.

    For callers that cannot allocate device memory at this point (see the header).  Nothing is
    allocated here either: ``beta_out`` (fp32, same shape as ``qw.beta``) comes from the caller.
    Raises QbloraError(ERR_TOO_LARGE) when (d_in/lambda_in)*(d_out/lambda_out) > 262144.
    """
    cq = qw.c_struct()
    ca = ad.c_struct()
    st = _lib.qablora_merge_noalloc(ctypes.byref(cq), ctypes.byref(ca), beta_out.data_ptr(), _stream_ptr(stream))
    _check(st, "qablora_merge_noalloc")
    return QWeight(qw.d_out, qw.d_in, qw.block_in, qw.block_out, qw.qfmt, qw.code, qw.codes, qw.alpha, beta_out, qw.code_bits)


def lowbit_gemm(qw: QWeight, X: torch.Tensor, out_dtype=torch.bfloat16, ws: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    assert X.is_cuda and X.is_contiguous() and X.dtype == torch.bfloat16
    T = X.shape[0]
    Y = out if out is not None else _empty((T, qw.d_out), out_dtype, X.device, stream)
    if ws is None:
        ws = alloc_workspace(OP_LOWBIT_GEMM, qw, None, T, stream)
    cq = qw.c_struct()
    st = _lib.qablora_lowbit_gemm(ctypes.byref(cq), X.data_ptr(), T, Y.data_ptr(), _dt(Y.dtype),
                                  ws.data_ptr(), ws.numel(), _stream_ptr(stream))
    _check(st, "qablora_lowbit_gemm")
    return Y


def dense_gemm(W: torch.Tensor, X: torch.Tensor, out_dtype=torch.bfloat16, ws: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """qblora_dense_gemm: Y = X W^T for a dense bf16 weight [d_out][d_in] (the merged 16-bit deployment)."""
    assert W.is_cuda and W.is_contiguous() and W.dtype == torch.bfloat16 and W.dim() == 2
    assert X.is_cuda and X.is_contiguous() and X.dtype == torch.bfloat16 and X.shape[1] == W.shape[1]
    T = X.shape[0]
    d_out, d_in = W.shape
    Y = out if out is not None else _empty((T, d_out), out_dtype, X.device, stream)
    if ws is None:
        ws = _empty(256, torch.uint8, X.device, stream)
    st = _lib.qblora_dense_gemm(W.data_ptr(), d_out, d_in, X.data_ptr(), T, Y.data_ptr(), _dt(Y.dtype), ws.data_ptr(),
                                ws.numel(), _stream_ptr(stream))
    _check(st, "qblora_dense_gemm")
    return Y


def pack_codes(qw: QWeight, bits: int, stream=None) -> QWeight:
    """qblora_pack_codes: the same weight with its codes in dense `bits`-bit storage (bits = 2 or 3)."""
    assert qw.code_bits == 4
    packed = _empty((qw.d_out, qw.d_in * bits // 8), torch.uint8, qw.codes.device, stream)
    ws = _empty(256, torch.uint8, qw.codes.device, stream)
    st = _lib.qblora_pack_codes(qw.codes.data_ptr(), qw.d_out, qw.d_in, int(bits), packed.data_ptr(), ws.data_ptr(), ws.numel(),
                                _stream_ptr(stream))
    _check(st, "qblora_pack_codes")
    _check(device_status(ws, stream), "qblora_pack_codes (a code does not fit)")
    return QWeight(qw.d_out, qw.d_in, qw.block_in, qw.block_out, qw.qfmt, qw.code, packed, qw.alpha, qw.beta, int(bits))


def unpack_codes(qw: QWeight, stream=None) -> QWeight:
    """qblora_unpack_codes: dense storage back to one code per nibble."""
    assert qw.code_bits in (2, 3)
    codes = _empty((qw.d_out, qw.d_in // 2), torch.uint8, qw.codes.device, stream)
    st = _lib.qblora_unpack_codes(qw.codes.data_ptr(), qw.d_out, qw.d_in, int(qw.code_bits), codes.data_ptr(), _stream_ptr(stream))
    _check(st, "qblora_unpack_codes")
    return QWeight(qw.d_out, qw.d_in, qw.block_in, qw.block_out, qw.qfmt, qw.code, codes, qw.alpha, qw.beta, 4)


# ------------------------------------------------------------------------------ between the products of a served layer
@dataclass
class Rope:
    """Rotary positions of a model: the first rotary_dim elements of every head are rotated, `table` from rope_table."""
    head_dim: int
    rotary_dim: int
    layout: int
    table: torch.Tensor              # int64 [rotary_dim / 2], device: turns per position in units of 2^-64
    amplitude: float = 1.0

    def c_struct(self) -> _CRope:
        t = self.table
        if t.dtype is not torch.int64 or not t.is_cuda or not t.is_contiguous() or 2 * t.numel() != self.rotary_dim:
            raise ValueError("table: contiguous int64 device tensor [rotary_dim / 2], see rope_table")
        return _CRope(self.head_dim, self.rotary_dim, self.layout, self.amplitude, t.data_ptr())


@dataclass
class KVCache:
    """Paged cache: k and v bf16 [n_pages][page_size][kv_heads][head_dim] (any order in memory: permuted views are fine
    as long as k and v agree and head_dim is contiguous)."""
    k: torch.Tensor
    v: torch.Tensor

    @staticmethod
    def empty(n_pages: int, page_size: int, kv_heads: int, head_dim: int, device="cuda") -> "KVCache":
        shape = (n_pages, page_size, kv_heads, head_dim)
        return KVCache(torch.empty(shape, dtype=torch.bfloat16, device=device),
                       torch.empty(shape, dtype=torch.bfloat16, device=device))

    def c_struct(self, sizes_only: bool = False) -> _CKVCache:
        k, v = self.k, self.v
        shape, stride = k.shape, k.stride()
        if len(shape) != 4 or shape != v.shape or stride != v.stride() or stride[3] != 1:
            raise ValueError("k, v: equal shapes and strides [n_pages][page_size][kv_heads][head_dim], head_dim contiguous")
        if k.dtype is not torch.bfloat16 or v.dtype is not torch.bfloat16 or not (sizes_only or k.is_cuda and v.is_cuda):
            raise ValueError("k, v: bf16 device tensors")
        return _CKVCache(k.data_ptr(), v.data_ptr(), stride[0], stride[1], stride[2], *shape)


@dataclass
class KVPlan:
    """Results of kv_plan (int32, device); see qblora_kv_plan."""
    cu_new: torch.Tensor             # [B + 1] first row of each request
    kv_len: torch.Tensor             # [B] cached tokens after the step
    positions: torch.Tensor          # [tokens]
    slots: torch.Tensor              # [tokens], -1 in unused rows
    admitted: torch.Tensor           # [B]
    free_count: torch.Tensor         # [1] pages left


def _heads(t: torch.Tensor) -> _CHeads:
    stride = t.stride()
    if len(stride) != 3 or stride[2] != 1 and t.shape[2] > 1 or not t.is_cuda:
        raise ValueError("[tokens][heads][head_dim] device tensor, head_dim contiguous")
    return _CHeads(t.data_ptr(), stride[0], stride[1], t.shape[1], _dt(t.dtype))


def _ints(t: torch.Tensor, n: int, name: str) -> int:
    if t.dtype is not torch.int32 or t.numel() < n or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name}: contiguous int32 device tensor of at least {n} entries")
    return t.data_ptr()


def rope_table(rotary_dim: int, base: float = 10000.0, scale: int = ROPE_SCALE_NONE, factor: float = 1.0,
               trained_len: int = 0, slow: float = 1.0, fast: float = 32.0, device="cuda") -> torch.Tensor:
    """qblora_rope_table: the rotation table of a model (int64 [rotary_dim / 2] on `device`)."""
    if rotary_dim < 2 or rotary_dim % 2:
        raise QbloraError(ERR_INVALID_ARG, "qblora_rope_table")
    buf = (ctypes.c_int64 * (rotary_dim // 2))()
    _check(_lib.qblora_rope_table(rotary_dim, base, scale, factor, trained_len, slow, fast, buf), "qblora_rope_table")
    return torch.tensor(list(buf), dtype=torch.int64, device=device)


def rope(cfg: Rope, positions: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor] = None, inverse: bool = False,
         out_q: Optional[torch.Tensor] = None, out_k: Optional[torch.Tensor] = None, stream=None):
    """qblora_rope on q (and k) [tokens][heads][head_dim]; inverse=True is the backward pass (gradients in, gradients
    out).  out_q / out_k may be q / k themselves.  Returns (q', k')."""
    shape, k_shape = q.shape, None if k is None else k.shape
    T, D = shape[0], cfg.head_dim
    if shape[2] != D or (k is not None and (k_shape[0] != T or k_shape[2] != D)):
        raise ValueError("q, k: [tokens][heads][head_dim]")
    if out_q is None:
        out_q = _empty(shape, q.dtype, q.device, stream)
    if k is not None and out_k is None:
        out_k = _empty(k_shape, out_q.dtype, k.device, stream)
    if out_q.shape != shape or (k is not None and out_k.shape != k_shape):
        raise ValueError("outputs have the shapes of the inputs")
    if T == 0:
        return out_q, out_k
    by = ctypes.byref
    st = _lib.qblora_rope(by(cfg.c_struct()), bool(inverse), _ints(positions, T, "positions"), T, by(_heads(q)), by(_heads(out_q)),
                          None if k is None else by(_heads(k)), None if k is None else by(_heads(out_k)), _stream_ptr(stream))
    if st != OK:
        _check(st, "qblora_rope")
    return out_q, out_k


def rope_append(cfg: Rope, positions: torch.Tensor, slots: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                cache: KVCache, out_q: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """qblora_rope_append: rotated q (bf16); rotated k and v go into the cache at `slots`."""
    shape, k_shape = q.shape, k.shape
    T, D = shape[0], cfg.head_dim
    if k_shape[0] != T or v.shape != k_shape or shape[2] != D or k_shape[2] != D:
        raise ValueError("q, k, v: [tokens][heads][head_dim]")
    if out_q is None:
        out_q = _empty(shape, torch.bfloat16, q.device, stream)
    elif out_q.shape != shape:
        raise ValueError("out_q has the shape of q")
    if T == 0:
        return out_q
    by = ctypes.byref
    st = _lib.qblora_rope_append(by(cfg.c_struct()), _ints(positions, T, "positions"), _ints(slots, T, "slots"), T, by(_heads(q)),
                                 by(_heads(k)), by(_heads(v)), by(_heads(out_q)), by(cache.c_struct()), _stream_ptr(stream))
    if st != OK:
        _check(st, "qblora_rope_append")
    return out_q


def kv_plan(ctx_len: torch.Tensor, new_len: torch.Tensor, block_table: torch.Tensor, free_pages: torch.Tensor,
            free_count: torch.Tensor, page_size: int, tokens: int, release: Optional[torch.Tensor] = None,
            outs: Optional[Tuple] = None, stream=None) -> KVPlan:
    """qblora_kv_plan: takes pages for the new tokens of every request (block_table and free_pages are updated in place)
    and returns the step's row offsets, lengths, positions and slots.  `tokens`: rows of the step's buffers.
    `outs`: preallocated (cu_new, kv_len, positions, slots, admitted, free_count)."""
    if block_table.dim() != 2:
        raise ValueError("block_table: [requests][width]")
    B, width = block_table.shape
    if outs is None:
        outs = tuple(_empty(n, torch.int32, block_table.device, stream) for n in (B + 1, B, tokens, tokens, B, 1))
    cu_new, kv_len, positions, slots, admitted, free_out = outs
    st = _lib.qblora_kv_plan(_ints(ctx_len, B, "ctx_len"), _ints(new_len, B, "new_len"),
                             None if release is None else _ints(release, B, "release"), B,
                             _ints(block_table, 1, "block_table"), width, _ints(free_pages, 1, "free_pages"),
                             free_pages.numel(), _ints(free_count, 1, "free_count"), _ints(free_out, 1, "free_count out"),
                             page_size, tokens, _ints(cu_new, B + 1, "cu_new"), _ints(kv_len, B, "kv_len"),
                             _ints(positions, tokens, "positions"), _ints(slots, tokens, "slots"),
                             _ints(admitted, B, "admitted"), _stream_ptr(stream))
    if st != OK:
        _check(st, "qblora_kv_plan")
    return KVPlan(cu_new, kv_len, positions, slots, admitted, free_out)


def attention_workspace_bytes(cache: KVCache, q_heads: int, tokens: int) -> int:
    c = cache.c_struct(sizes_only=True)
    return int(_lib.qblora_attention_workspace_bytes(ctypes.byref(c), q_heads, tokens))


def alloc_attention_workspace(cache: KVCache, q: torch.Tensor, stream=None) -> torch.Tensor:
    """Workspace for paged_attention calls (on `stream`) with this cache and up to q.shape[0] tokens."""
    n = max(attention_workspace_bytes(cache, q.shape[1], max(q.shape[0], 1)), 256)
    return _empty(n, torch.uint8, q.device, stream)


def paged_attention(q: torch.Tensor, cache: KVCache, block_table: torch.Tensor, cu_new: torch.Tensor, kv_len: torch.Tensor,
                    scale: Optional[float] = None, causal: bool = True, window: int = 0, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, need_lse: bool = False, ws: Optional[torch.Tensor] = None, stream=None):
    """qblora_paged_attention: q bf16 [tokens][q_heads][head_dim] -> (out, lse); lse (fp32 [tokens][q_heads]) is None
    unless need_lse or a tensor for it is given.  scale defaults to head_dim^-1/2; window = 0: no window."""
    shape = q.shape
    T, H, D = shape
    cc = cache.c_struct()
    if D != cc.head_dim:
        raise ValueError("q: [tokens][q_heads][head_dim of the cache]")
    B, width = block_table.shape
    if out is None:
        out = _empty(shape, torch.bfloat16, q.device, stream)
    if lse is None and need_lse:
        lse = _empty((T, H), torch.float32, q.device, stream)
    if out.shape != shape or (lse is not None and (lse.shape != (T, H) or lse.dtype is not torch.float32 or not lse.is_contiguous() or not lse.is_cuda)):
        raise ValueError("out: shape of q; lse: contiguous fp32 device tensor [tokens][q_heads]")
    if T == 0:
        return out, lse
    if ws is None:
        ws = alloc_attention_workspace(cache, q, stream)
    elif not ws.is_cuda or ws.dtype is not torch.uint8 or not ws.is_contiguous():
        raise ValueError("ws: contiguous uint8 device tensor")
    by = ctypes.byref
    st = _lib.qblora_paged_attention(by(cc), _ints(block_table, 1, "block_table"), width, _ints(cu_new, B + 1, "cu_new"),
                                     _ints(kv_len, B, "kv_len"), B, by(_heads(q)), T, D ** -0.5 if scale is None else scale,
                                     bool(causal), window, by(_heads(out)), None if lse is None else lse.data_ptr(),
                                     ws.data_ptr(), ws.numel(), _stream_ptr(stream))
    if st != OK:
        _check(st, "qblora_paged_attention")
    return out, lse

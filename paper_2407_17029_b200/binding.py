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
           "qblora_paged_attention",
           "qblora_adapter_plan", "qblora_adapters_workspace_bytes", "qblora_adapters_fwd", "qblora_adapters_bwd",
           "qblora_adamw_workspace_bytes", "qblora_adamw_prepare", "qblora_adamw_step"]


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


class _CAdapterBank(ctypes.Structure):
    _fields_ = [("d_in", ctypes.c_int32), ("d_out", ctypes.c_int32), ("lambda_in", ctypes.c_int32), ("lambda_out", ctypes.c_int32),
                ("n_adapters", ctypes.c_int32), ("rank", ctypes.c_int32), ("A", ctypes.c_void_p), ("B", ctypes.c_void_p),
                ("scaling", ctypes.c_void_p), ("ranks", ctypes.c_void_p)]


class _CAdamWTensor(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("g", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("g_dtype", ctypes.c_int32), ("state_bits", ctypes.c_int32), ("lr_mult", ctypes.c_float),
                ("weight_decay", ctypes.c_float)]


class _CAdamWCfg(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_void_p), ("steps", ctypes.c_void_p), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("max_norm", ctypes.c_double), ("seed", ctypes.c_uint32), ("norm", ctypes.c_void_p)]


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
_lib.qblora_adapter_plan.argtypes = [_vp, _vp, _i32, _i32, _i64, _vp, _vp, _vp]
_lib.qblora_adapters_workspace_bytes.restype = _sz
_lib.qblora_adapters_workspace_bytes.argtypes = [_vp, _i64, ctypes.c_int]
_lib.qblora_adapters_fwd.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _vp, _i64, ctypes.c_int, _vp, _sz, _vp]
_lib.qblora_adapters_bwd.argtypes = [_vp, _vp, _vp, _vp, _i64, _vp, _i64, _i64, _vp, _i64, ctypes.c_int, _vp, _vp, _vp, _sz, _vp]
_lib.qblora_adamw_workspace_bytes.restype = _sz
_lib.qblora_adamw_workspace_bytes.argtypes = [_i32]
_lib.qblora_adamw_prepare.argtypes = [_vp, _i32, _vp, _sz, _vp, _vp]
_lib.qblora_adamw_step.argtypes = [_vp, _i32, _i64, _vp, _sz, _vp]


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


_current_device = _raw_device if _raw_device is not None else torch.cuda.current_device


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


# ------------------------------------------------------------------------------------ many adapters over one frozen weight
@dataclass
class AdapterBank:
    """Adapters of one layer, a slot each: A bf16 [n][P][rank], B bf16 [n][rank][Q], scaling fp32 [n] (device, contiguous).
    An adapter of a lower rank has zeros behind it; `ranks` (int32 [n]) saves the work on them."""
    d_in: int
    d_out: int
    lambda_in: int
    lambda_out: int
    A: torch.Tensor
    B: torch.Tensor
    scaling: torch.Tensor
    ranks: Optional[torch.Tensor] = None

    def c_struct(self) -> _CAdapterBank:
        A, B, s, k = self.A, self.B, self.scaling, self.ranks
        if self.lambda_in < 1 or self.lambda_out < 1 or A.dim() != 3:
            raise ValueError("lambda_in, lambda_out >= 1; A: [n][d_in / lambda_in][rank]")
        n, P, r = A.shape
        if P * self.lambda_in != self.d_in or B.shape != (n, r, self.d_out // self.lambda_out) or B.shape[2] * self.lambda_out != self.d_out:
            raise ValueError("A: [n][d_in / lambda_in][rank], B: [n][rank][d_out / lambda_out]")
        at = A.get_device()
        if A.dtype is not torch.bfloat16 or B.dtype is not torch.bfloat16 or not (A.is_contiguous() and B.is_contiguous()) or at < 0 or B.get_device() != at:
            raise ValueError("A, B: contiguous bf16 device tensors")
        if s.dtype is not torch.float32 or s.numel() != n or not s.is_contiguous() or s.get_device() != at:
            raise ValueError("scaling: contiguous fp32 device tensor [n]")
        return _CAdapterBank(self.d_in, self.d_out, self.lambda_in, self.lambda_out, n, r, A.data_ptr(), B.data_ptr(), s.data_ptr(),
                             None if k is None else _ints_at(k, n, "ranks", at))


def _elsewhere(t: torch.Tensor):
    """t.get_device() is not the current device, where a call's kernels run."""
    raise ValueError(f"tensors on the current device (there are some on {t.device})")


def _ints_at(t: torch.Tensor, n: int, name: str, at: int) -> int:
    if t.dtype is not torch.int32 or t.numel() < n or not t.is_contiguous() or t.get_device() != at:
        raise ValueError(f"{name}: contiguous int32 tensor of at least {n} entries on the other tensors' device")
    return t.data_ptr()


@dataclass
class AdapterPlan:
    """Rows of a step sorted by adapter (int32, device); see qblora_adapter_plan."""
    rows: torch.Tensor               # [tokens] row numbers, -1 behind the last one
    start: torch.Tensor              # [n_adapters + 1] first entry of each adapter


def adapter_plan(cu_rows: torch.Tensor, adapter_ids: torch.Tensor, n_adapters: int, tokens: int, outs: Optional[Tuple] = None,
                 stream=None) -> AdapterPlan:
    """qblora_adapter_plan: request b has the rows cu_rows[b] .. cu_rows[b + 1] - 1 and uses adapter_ids[b] (-1: none).
    `tokens`: rows of the step's buffers.  `outs`: preallocated (rows, start)."""
    B, at = adapter_ids.numel(), adapter_ids.get_device()
    if at < 0 or at != _current_device():
        _elsewhere(adapter_ids)
    rows, start = outs if outs is not None else (_empty(n, torch.int32, adapter_ids.device, stream) for n in (tokens, n_adapters + 1))
    st = _lib.qblora_adapter_plan(_ints_at(cu_rows, B + 1, "cu_rows", at), _ints_at(adapter_ids, B, "adapter_ids", at), B, n_adapters, tokens,
                                  _ints_at(rows, tokens, "rows", at), _ints_at(start, n_adapters + 1, "start", at), _stream_ptr(stream))
    if st != OK:
        _check(st, "qblora_adapter_plan")
    return AdapterPlan(rows, start)


def _rows(t: torch.Tensor, tokens: int, width: int, name: str, at: int, dtypes=(torch.bfloat16,)) -> int:
    """Checks a [tokens][width] tensor with contiguous rows on device `at`; returns its row stride."""
    if t.shape != (tokens, width) or t.get_device() != at or t.dtype not in dtypes:
        raise ValueError(f"{name}: [{tokens}][{width}] tensor on the bank's device, of {' or '.join(str(d) for d in dtypes)}")
    step, one = t.stride()
    if (one != 1 and width > 1) or (step < width and tokens > 1):
        raise ValueError(f"{name}: rows are contiguous and do not overlap")
    return step if step > width else width


def adapters_workspace_bytes(bank: AdapterBank, tokens: int, backward: bool = False) -> int:
    return int(_lib.qblora_adapters_workspace_bytes(ctypes.byref(bank.c_struct()), tokens, bool(backward)))


def alloc_adapters_workspace(bank: AdapterBank, tokens: int, backward: bool = False, stream=None) -> torch.Tensor:
    """Workspace for adapters_fwd (or adapters_bwd) calls (on `stream`) with banks of this size and up to `tokens` rows."""
    return _empty(max(adapters_workspace_bytes(bank, max(tokens, 1), backward), 256), torch.uint8, bank.A.device, stream)


def _workspace(ws: torch.Tensor, at: int) -> torch.Tensor:
    if ws.get_device() != at or ws.dtype is not torch.uint8 or not ws.is_contiguous():
        raise ValueError("ws: contiguous uint8 tensor on the bank's device")
    return ws


def adapters_fwd(bank: AdapterBank, plan: AdapterPlan, X: torch.Tensor, Y: torch.Tensor, ws: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
    """qblora_adapters_fwd: adds every planned row's adapter term to Y [tokens][d_out] (bf16 or fp32, what the shared
    projection of X has written) in place; returns Y.  X and Y have the `tokens` rows that the plan was made for."""
    T, at = X.shape[0], bank.A.get_device()
    if at < 0 or at != _current_device():
        _elsewhere(bank.A)
    xs = _rows(X, T, bank.d_in, "X", at)
    ys = _rows(Y, T, bank.d_out, "Y", at, (torch.bfloat16, torch.float32))
    c = bank.c_struct()
    if T == 0:
        return Y
    ws = alloc_adapters_workspace(bank, T, stream=stream) if ws is None else _workspace(ws, at)
    st = _lib.qblora_adapters_fwd(ctypes.byref(c), _ints_at(plan.rows, T, "rows", at), _ints_at(plan.start, c.n_adapters + 1, "start", at), X.data_ptr(),
                                  xs, T, Y.data_ptr(), ys, _dt(Y.dtype), ws.data_ptr(), ws.numel(), _stream_ptr(stream))
    if st != OK:
        _check(st, "qblora_adapters_fwd")
    return Y


def adapters_bwd(bank: AdapterBank, plan: AdapterPlan, X: Optional[torch.Tensor], dY: torch.Tensor, dX: Optional[torch.Tensor] = None,
                 need_da: bool = True, need_db: bool = True, outs: Optional[Tuple] = None, ws: Optional[torch.Tensor] = None,
                 stream=None):
    """qblora_adapters_bwd: adds the adapters' part to dX [tokens][d_in] (bf16 or fp32, what the shared projection's backward
    pass has written; None: not wanted) in place and returns (dX, dA, dB), dA and dB fp32 of the shapes of A and B.
    `outs`: preallocated (dA, dB), entries None where not wanted."""
    T, at = dY.shape[0], bank.A.get_device()
    if at < 0 or at != _current_device():
        _elsewhere(bank.A)
    ds = _rows(dY, T, bank.d_out, "dY", at)
    c = bank.c_struct()
    if outs is not None:
        dA, dB = outs
        for g, like, name in ((dA, bank.A, "dA"), (dB, bank.B, "dB")):
            if g is not None and (g.shape != like.shape or g.dtype is not torch.float32 or not g.is_contiguous() or g.get_device() != at):
                raise ValueError(f"{name}: contiguous fp32 device tensor of the shape of {name[1]}")
    else:
        dA = _empty(bank.A.shape, torch.float32, dY.device, stream) if need_da else None
        dB = _empty(bank.B.shape, torch.float32, dY.device, stream) if need_db else None
    gs = _rows(dX, T, bank.d_in, "dX", at, (torch.bfloat16, torch.float32)) if dX is not None else 0
    xs = _rows(X, T, bank.d_in, "X", at) if X is not None else 0
    if T == 0:
        for g in (dA, dB):
            if g is not None:
                _zero(g, stream)
        return dX, dA, dB
    ws = alloc_adapters_workspace(bank, T, backward=True, stream=stream) if ws is None else _workspace(ws, at)
    p = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    st = _lib.qblora_adapters_bwd(ctypes.byref(c), _ints_at(plan.rows, T, "rows", at), _ints_at(plan.start, c.n_adapters + 1, "start", at), p(X), xs,
                                  dY.data_ptr(), ds, T, p(dX), gs, _dt(dX.dtype) if dX is not None else BF16, p(dA), p(dB),
                                  ws.data_ptr(), ws.numel(), _stream_ptr(stream))
    if st != OK:
        _check(st, "qblora_adapters_bwd")
    return dX, dA, dB


class _Order:
    """Calls that share buffers, one behind the other whatever streams they are on; called with a call's stream it gives the handle.
    `tensors`: memory of the first stream, which the others use too."""

    def __init__(self, tensors=()):
        self._handle, self._stream, self._tensors = None, None, tensors

    def __call__(self, stream) -> int:
        handle = _stream_ptr(stream)
        if handle != self._handle:
            self._change(stream if stream is not None else torch.cuda.current_stream(), handle)
        return handle

    def _change(self, stream, handle) -> None:
        if _capturing(stream):              # nothing runs now, and a graph cannot wait for work outside
            return
        if self._stream is not None:
            if _capturing(self._stream):
                raise RuntimeError("the stream of the call before is being captured: order the two streams when that has ended")
            stream.wait_stream(self._stream)
            for t in self._tensors:
                t.record_stream(stream)
        self._handle, self._stream = handle, stream


def _capturing(stream) -> bool:
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


def _zero(t: torch.Tensor, stream) -> None:
    if stream is None:
        t.zero_()
    else:
        with torch.cuda.stream(stream):
            t.zero_()


class AdamW:
    """qblora_adamw_step over a list of tensors; the table of their addresses is made here, once.

    params fp32, grads fp32 or bf16, copies (optional) bf16: lists of contiguous device tensors of equal sizes; an entry of copies may
    be None.  state_bits 32 or 8 (or a list): states m, v are fp32 tensors, or float8_e4m3fn codes of the first average and of
    the second one's square root with one fp32 scale per 256 elements in m_scale, v_scale.  They start at zero; `states` takes
    kept ones (a dict of lists with these names), `steps` a kept count (int32 [1], device).  lr: a number, or an fp32 device tensor [1]
    that a schedule writes; lr_mult and weight_decay: numbers or lists.  max_norm > 0 clips by the global norm, need_norm asks
    for it alone (self.norm, fp32 [1]).

    The constructor, set_grads and step share the table: each of them waits, on its own stream, for the one before it, whatever stream that
    was on.  A step that is captured waits for nothing and nothing waits for it: its graph is replayed behind the constructor and the
    last set_grads, and not beside another step."""

    def __init__(self, params, grads, copies=None, state_bits=32, states=None, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay=0.0, lr_mult=1.0, max_norm: float = 0.0, need_norm: bool = False, seed: int = 0, steps=None, stream=None):
        n = len(params)
        if n < 1 or len(grads) != n or (copies is not None and len(copies) != n):
            raise ValueError("params, grads, copies: lists of equal length, at least one tensor")
        each = lambda x: list(x) if isinstance(x, (list, tuple)) else [x] * n  # noqa: E731
        bits, decay, mult = each(state_bits), each(weight_decay), each(lr_mult)
        if len(bits) != n or len(decay) != n or len(mult) != n or any(b not in (8, 32) for b in bits):
            raise ValueError("state_bits (8 or 32), weight_decay, lr_mult: a value, or a list with one for each tensor")
        self._index = params[0].get_device()
        if self._index < 0 or self._index != _current_device():
            _elsewhere(params[0])
        self.device = params[0].device
        self.params, self.grads, self.copies = list(params), list(grads), list(copies) if copies is not None else [None] * n
        new = lambda shape, dtype: _zeros(shape, dtype, self.device, stream)  # noqa: E731
        blocks = [(p.numel() + 255) // 256 for p in self.params]
        states = states or {}
        make = {"m": lambda k: new(self.params[k].shape, torch.float32 if bits[k] == 32 else torch.float8_e4m3fn),
                "m_scale": lambda k: new((blocks[k],), torch.float32) if bits[k] == 8 else None}
        make["v"], make["v_scale"] = make["m"], make["m_scale"]
        if any(k not in make or len(v) != n for k, v in states.items()):
            raise ValueError("states: lists named m, v, m_scale, v_scale with an entry for each tensor")
        self.m, self.v, self.m_scale, self.v_scale = ([states[name][k] if states.get(name) is not None else make[name](k) for k in range(n)]
                                                      for name in ("m", "v", "m_scale", "v_scale"))
        self.steps = steps if steps is not None else new((1,), torch.int32)
        if not isinstance(lr, torch.Tensor):
            value, lr = float(lr), new((1,), torch.float32)
            with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream(self.device)):
                lr.fill_(value)
        self.lr = lr
        self.norm = new((1,), torch.float32) if need_norm or max_norm > 0 else None
        for t, dtype, name in ((self.steps, torch.int32, "steps"), (self.lr, torch.float32, "lr")):
            if t.dtype is not dtype or t.numel() != 1 or t.device != self.device or not t.is_cuda:
                raise ValueError(f"{name}: {dtype} tensor [1] on the parameters' device")
        table = (_CAdamWTensor * n)()
        for k in range(n):
            size = self.params[k].numel()
            state = torch.float32 if bits[k] == 32 else torch.float8_e4m3fn
            for t, dtypes, count, name in ((self.params[k], (torch.float32,), size, "params"), (self.grads[k], (torch.float32, torch.bfloat16), size, "grads"),
                                           (self.copies[k], (torch.bfloat16, None), size, "copies"), (self.m[k], (state,), size, "m"), (self.v[k], (state,), size, "v"),
                                           (self.m_scale[k] if bits[k] == 8 else None, (torch.float32, None) if bits[k] == 32 else (torch.float32,), blocks[k], "m_scale"),
                                           (self.v_scale[k] if bits[k] == 8 else None, (torch.float32, None) if bits[k] == 32 else (torch.float32,), blocks[k], "v_scale")):
                if t is None and None in dtypes:
                    continue
                if t is None or t.dtype not in dtypes or t.numel() != count or not t.is_contiguous() or t.device != self.device or not t.is_cuda:
                    raise ValueError(f"{name}[{k}]: contiguous {dtypes[0]} tensor of {count} elements on the parameters' device")
            p = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
            table[k] = _CAdamWTensor(p(self.params[k]), p(self.grads[k]), p(self.copies[k]), p(self.m[k]), p(self.v[k]),
                                     p(self.m_scale[k]) if bits[k] == 8 else None, p(self.v_scale[k]) if bits[k] == 8 else None, size,
                                     _dt(self.grads[k].dtype), bits[k], mult[k], decay[k])
        self._n, self._blocks, self._table = n, ctypes.c_int64(), table
        made = [t for t in (self.steps if steps is None else None, self.lr, self.norm) if t is not None]
        made += [t for name in make for k, t in enumerate(getattr(self, name)) if t is not None and states.get(name) is None]
        self.ws = _empty(max(int(_lib.qblora_adamw_workspace_bytes(n)), 256), torch.uint8, self.device, stream)
        self._cfg = _CAdamWCfg(self.lr.data_ptr(), self.steps.data_ptr(), float(betas[0]), float(betas[1]), float(eps), float(max_norm),
                               int(seed) & 0xffffffff, p(self.norm))
        self._order = _Order([self.ws] + made)
        self._prepare(stream)

    def _prepare(self, stream):
        if self._index != _current_device():
            _elsewhere(self.ws)
        _check(_lib.qblora_adamw_prepare(self._table, self._n, self.ws.data_ptr(), self.ws.numel(), ctypes.byref(self._blocks), self._order(stream)),
               "qblora_adamw_prepare")

    def set_grads(self, grads, stream=None) -> None:
        """Other gradient tensors from the next step on (a new table: about 0.5 ms of the host's time for 560 tensors, so a training loop had better
        keep its gradients' tensors; not while a captured step of this object may run)."""
        if len(grads) != self._n:
            raise ValueError("grads: one tensor for each parameter")
        for k, g in enumerate(grads):
            if g.dtype not in (torch.float32, torch.bfloat16) or g.numel() != self.params[k].numel() or not g.is_contiguous() or g.device != self.device:
                raise ValueError(f"grads[{k}]: contiguous fp32 or bf16 tensor of the parameter's size and device")
        for k, g in enumerate(grads):
            self._table[k].g, self._table[k].g_dtype = g.data_ptr(), _dt(g.dtype)
        self.grads = list(grads)
        self._prepare(stream)

    def step(self, stream=None) -> Optional[torch.Tensor]:
        """One step on the gradients as they are when it runs; returns the norm's tensor, where it is formed."""
        if self._index != _current_device():
            _elsewhere(self.ws)
        st = _lib.qblora_adamw_step(ctypes.byref(self._cfg), self._n, self._blocks.value, self.ws.data_ptr(), self.ws.numel(), self._order(stream))
        if st != OK:
            _check(st, "qblora_adamw_step")
        return self.norm


def _zeros(shape, dtype, device, stream) -> torch.Tensor:
    t = _empty(shape, torch.uint8 if dtype is torch.float8_e4m3fn else dtype, device, stream)
    _zero(t, stream)
    return t.view(dtype) if dtype is torch.float8_e4m3fn else t

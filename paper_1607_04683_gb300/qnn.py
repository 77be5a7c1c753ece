"""Thin Python binding of libqnn (include/qnn.h) with the same call names.

Argument marshalling only: every step of the computation runs in the CUDA library. PyTorch
provides device memory and the current stream. If libqnn.so is missing or cannot be loaded the
calls raise; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libqnn.so")

QNN_OK = 0
QNN_ERR_INVALID_ARG = 1
QNN_ERR_NONFINITE = 2
QNN_ERR_K_TOO_LARGE = 3
QNN_ERR_CUDA = 4
QNN_ERR_TIMEOUT = 5
QNN_ERR_NO_COOP = 6
QNN_ERR_NO_MEMORY = 7
PER_MATRIX, PER_ROW = 0, 1
OUT_NONE, OUT_QUANT, OUT_FLOAT = 0, 1, 2
K_MAX = 33025

# qnn_qparams {float vmin, vmax, Q; int32 z} as a numpy record (16 bytes)
QPARAMS_DTYPE = np.dtype([("vmin", "<f4"), ("vmax", "<f4"), ("Q", "<f4"), ("z", "<i4")])

# Every symbol the header declares (checked by the CPU test that loads the library).
EXPORTS = ("qnn_status_string", "qnn_device_status", "qnn_quantize", "qnn_qmatmul", "qnn_lstm_param_count",
           "qnn_lstm_model_create", "qnn_lstm_model_destroy", "qnn_lstm_model_weights", "qnn_lstm_forward",
           "qnn_lstm_forward_logits",
           "qnn_profile_enable", "qnn_profile_read", "qnn_measure_peak", "qnn_quantize_matrix_static",
           "qnn_selftest_s64_to_f32", "qnn_stack_frames", "qnn_selftest_wait_timeout", "qnn_selftest_pair_functions", "qnn_lstm_stream_open",
           "qnn_lstm_stream_push", "qnn_lstm_stream_pull", "qnn_lstm_stream_close", "qnn_measure_exchange_floor",
           "qnn_rmsnorm_quantize", "qnn_quantize4", "qnn_qmatmul4", "qnn_causal_conv", "qnn_ssm_scan")

_DTYPES = {}  # qnn_dtype of a torch type
_MOST_SUMMED = (2 ** 31 - 1) // 255  # values of a row whose codes' sum has 32 bits
# qnn_ssm_args as it lies in memory
_SSM_ARGS = struct.Struct("=3q4i" + 6 * "Q2q" + "6Q")


class QnnError(RuntimeError):
    def __init__(self, status: int, where: str = ""):
        self.status = status
        msg = lib().qnn_status_string(status).decode() if _lib is not None else f"status {status}"
        super().__init__(f"{where}: {msg}" if where else msg)


class LstmDesc(C.Structure):
    _fields_ = [("num_layers", C.c_int32), ("input_dim", C.c_int32), ("hidden", C.c_int32),
                ("proj", C.c_int32), ("num_classes", C.c_int32), ("output_mode", C.c_int32),
                ("stack", C.c_int32), ("stack_stride", C.c_int32), ("weight_blocks", C.c_int32)]


class SsmArgs(C.Structure):
    """qnn_ssm_args"""
    _fields_ = [("B", C.c_int64), ("T", C.c_int64), ("D", C.c_int64), ("N", C.c_int32), ("groups", C.c_int32),
                ("dtype", C.c_int32), ("softplus", C.c_int32),
                *[(n + f, C.c_void_p if f == "" else C.c_int64) for n in ("u", "dt", "Bm", "Cm", "z", "y")
                  for f in ("", "_seq", "_frame")],
                ("A", C.c_void_p), ("skip", C.c_void_p), ("dt_bias", C.c_void_p), ("state_in", C.c_void_p),
                ("state_out", C.c_void_p), ("lengths", C.c_void_p)]


_lib = None


def lib():
    """Load libqnn.so (build it first with __graft_entry__.build() or paper_1607_04683_gb300.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libqnn.so not built at {LIB_PATH}; run the package build first")
        L = C.CDLL(LIB_PATH)
        P, i64, i32 = C.c_void_p, C.c_int64, C.c_int
        L.qnn_status_string.argtypes = [i32]
        L.qnn_status_string.restype = C.c_char_p
        L.qnn_device_status.argtypes = [P]
        L.qnn_device_status.restype = i32
        L.qnn_quantize.argtypes = [P, i64, i64, i64, i32, P, i64, P, P, P]
        L.qnn_quantize.restype = i32
        L.qnn_qmatmul.argtypes = [P, i64, P, i32, P, i64, i64, P, i64, P, i64, P, i64, P, P, i64, P, P]
        L.qnn_qmatmul.restype = i32
        L.qnn_lstm_param_count.argtypes = [C.POINTER(LstmDesc)]
        L.qnn_lstm_param_count.restype = i64
        L.qnn_lstm_model_create.argtypes = [C.POINTER(LstmDesc), P, C.POINTER(P)]
        L.qnn_lstm_model_create.restype = i32
        L.qnn_lstm_model_destroy.argtypes = [P]
        L.qnn_lstm_model_destroy.restype = None
        L.qnn_lstm_model_weights.argtypes = [P, P, P, C.POINTER(i64)]
        L.qnn_lstm_model_weights.restype = i32
        L.qnn_lstm_forward.argtypes = [P, P, i64, i64, P, P, P, P, P]
        L.qnn_lstm_forward.restype = i32
        L.qnn_lstm_forward_logits.argtypes = [P, P, i64, i64, P, P, P, P, P, P]
        L.qnn_lstm_forward_logits.restype = i32
        L.qnn_profile_enable.argtypes = [i32]
        L.qnn_profile_enable.restype = i32
        L.qnn_profile_read.argtypes = [i32, P, P, P, C.POINTER(i32)]
        L.qnn_profile_read.restype = i32
        L.qnn_measure_peak.argtypes = [i32, C.POINTER(C.c_double)]
        L.qnn_measure_peak.restype = i32
        L.qnn_selftest_s64_to_f32.argtypes = [P, P, i64, P]
        L.qnn_stack_frames.argtypes = [P, i64, i64, i64, i32, i32, P, P]
        L.qnn_selftest_pair_functions.argtypes = [P, i64, P, P]
        L.qnn_selftest_pair_functions.restype = i32
        L.qnn_selftest_wait_timeout.argtypes = [i64, P]
        L.qnn_selftest_wait_timeout.restype = i32
        L.qnn_stack_frames.restype = i32
        L.qnn_selftest_s64_to_f32.restype = i32
        L.qnn_measure_exchange_floor.argtypes = [i32, i32, C.POINTER(C.c_double)]
        L.qnn_measure_exchange_floor.restype = i32
        L.qnn_lstm_stream_open.argtypes = [P, i64, i64, C.c_double, C.POINTER(P)]
        L.qnn_lstm_stream_open.restype = i32
        L.qnn_lstm_stream_push.argtypes = [P, P, i64]
        L.qnn_lstm_stream_push.restype = i32
        L.qnn_lstm_stream_pull.argtypes = [P, P, i64, C.c_double]
        L.qnn_lstm_stream_pull.restype = i32
        L.qnn_lstm_stream_close.argtypes = [P]
        L.qnn_lstm_stream_close.restype = i32
        L.qnn_quantize_matrix_static.argtypes = [P, i64, i64, i64, P, i64, P, P, P, P]
        L.qnn_quantize_matrix_static.restype = i32
        L.qnn_rmsnorm_quantize.argtypes = [P, i64, P, i64, i32, P, C.c_double, i64, i64, P, i64, P, i64, P, P, P, i64, P]
        L.qnn_rmsnorm_quantize.restype = i32
        L.qnn_quantize4.argtypes = [P, i64, i64, i64, C.c_int32, P, P, P, P]
        L.qnn_quantize4.restype = i32
        L.qnn_qmatmul4.argtypes = [P, i64, P, i32, i64, i64, P, P, C.c_int32, P, i64, P, P, i64, P]
        L.qnn_qmatmul4.restype = i32
        L.qnn_causal_conv.argtypes = [P, i64, i64, i32, i64, i64, i64, P, C.c_int32, P, i32, P, P, P, P, i64, i64, P]
        L.qnn_causal_conv.restype = i32
        L.qnn_ssm_scan.argtypes = [P, P]
        L.qnn_ssm_scan.restype = i32
        _lib = L
    return _lib


def profile_enable(on: bool = True):
    _check(lib().qnn_profile_enable(1 if on else 0), "qnn_profile_enable")


def measure_peak(kind: int) -> float:
    """Measured peak TOPS of an integer datapath: 0 = mma.sync u8 tensor-core MMA, 1 = dp4a."""
    v = C.c_double(0.0)
    _check(lib().qnn_measure_peak(kind, C.byref(v)), "qnn_measure_peak")
    return v.value


def measure_exchange_floor(cluster_size: int, rounds: int = 20000) -> float:
    """Microseconds per round of the batch-of-few recurrence's per-frame synchronisation skeleton
    (no arithmetic) on one cluster of cluster_size blocks: the floor under a layer's time per frame."""
    v = C.c_double(0.0)
    _check(lib().qnn_measure_exchange_floor(cluster_size, rounds, C.byref(v)), "qnn_measure_exchange_floor")
    return v.value


def selftest_s64_to_f32(values):
    """The device's int64 -> fp32 round-to-nearest conversion of the recovery, on a torch int64
    CUDA tensor; returns a float32 tensor (diagnostic)."""
    import torch
    out = torch.empty(values.shape, dtype=torch.float32, device=values.device)
    _check(lib().qnn_selftest_s64_to_f32(values.data_ptr(), out.data_ptr(), values.numel(),
                                         torch.cuda.current_stream().cuda_stream), "qnn_selftest_s64_to_f32")
    return out


def selftest_pair_functions(values) -> int:
    """Pairs of a float32 CUDA tensor through the gate kernel's paired-instruction functions and
    their one-value forms; returns the number of pairs whose results differ in any bit."""
    import torch
    out = torch.zeros(1, dtype=torch.int64, device=values.device)
    _check(lib().qnn_selftest_pair_functions(values.data_ptr(), values.numel() // 2, out.data_ptr(),
                                             torch.cuda.current_stream().cuda_stream), "qnn_selftest_pair_functions")
    return int(out.item())


def selftest_wait_timeout(limit_ns: int, stream=None):
    """A bounded device wait that nothing ends: raises unless it gave up as designed."""
    _check(lib().qnn_selftest_wait_timeout(int(limit_ns), _stream(stream)), "qnn_selftest_wait_timeout")


def profile_read() -> dict:
    """{kernel name: (launches, total device ms)} since the last read (waits for the events)."""
    cap = 64
    names = (C.c_char_p * cap)()
    ms = (C.c_double * cap)()
    n_l = (C.c_int64 * cap)()
    cnt = C.c_int(0)
    _check(lib().qnn_profile_read(cap, C.cast(names, C.c_void_p), C.cast(ms, C.c_void_p), C.cast(n_l, C.c_void_p),
                                  C.byref(cnt)), "qnn_profile_read")
    return {names[i].decode(): (int(n_l[i]), float(ms[i])) for i in range(min(cnt.value, cap))}


def _check(st: int, where: str):
    if st != QNN_OK:
        raise QnnError(st, where)


def _p(t):
    """Raw pointer of a torch tensor or numpy array (None -> NULL)."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data_as(C.c_void_p)
    return t.data_ptr()


def _stream(stream):
    """Raw handle of stream, or of the current stream of the current device. A product of one frame is bound
    by the host: 13.5 us of its time a call with a Stream object and wrapped pointers made for each call, 7.5 us
    without (a result passed in; 14 to 17 us a call with one allocated, 2048 x 2048)."""
    if stream is not None:
        return stream.cuda_stream
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


_torch = None


def _libs():
    """torch and the library, for the calls whose marshalling is most of their time."""
    global _torch
    if _torch is None:
        import torch
        torch.cuda.current_device()  # (starts CUDA)
        _torch = torch
        _DTYPES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    return _torch, _lib or lib()


def _here(torch):
    """The current stream of the current device (half of _stream's time)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def params_view(p) -> np.ndarray:
    """Device params tensor (int32 [n, 4]) -> numpy records with fields vmin, vmax, Q, z."""
    return p.detach().cpu().numpy().view(QPARAMS_DTYPE).reshape(-1)


def params_tensor(records: np.ndarray, device="cuda"):
    import torch
    raw = np.ascontiguousarray(records, QPARAMS_DTYPE).view(np.int32).reshape(-1, 4)
    return torch.from_numpy(raw.copy()).to(device)


def device_status(stream=None) -> int:
    return int(lib().qnn_device_status(_stream(stream)))


def qnn_quantize(x, granularity=PER_MATRIX, stream=None):
    """x: CUDA fp32 [rows, cols] (row stride may exceed cols). Returns (codes u8, params int32 [n,4],
    code_sums int32 [rows])."""
    import torch
    assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1
    rows, cols = x.shape
    codes = torch.empty((rows, cols), dtype=torch.uint8, device=x.device)
    # every unit is written, but for a call without rows
    params = (torch.empty if rows else torch.zeros)((1 if granularity == PER_MATRIX else rows, 4), dtype=torch.int32,
                                                    device=x.device)
    sums = torch.empty(rows, dtype=torch.int32, device=x.device)
    _check(lib().qnn_quantize(_p(x), rows, cols, x.stride(0), granularity, _p(codes), cols, _p(params), _p(sums),
                              _stream(stream)), "qnn_quantize")
    return codes, params, sums


def qnn_qmatmul(A, pa, ga, rsA, W, pw, csW, n_blocks=1, bias=None, want_acc=False, out=None, stream=None):
    """Y = R(A' W'^T) + bias (eq. 1). A u8 [M, K], W u8 [N, K] (CUDA). Returns (Y fp32 [M, N], acc or None)."""
    import torch
    M, K = A.shape
    N, K2 = W.shape
    (lda, a1), (ldw, w1) = A.stride(), W.stride()
    assert K == K2 and a1 == 1 and w1 == 1
    Y = out if out is not None else torch.empty((M, N), dtype=torch.float32, device=A.device)
    acc = torch.empty((M, N), dtype=torch.int32, device=A.device) if want_acc else None
    _check(lib().qnn_qmatmul(_p(A), lda, _p(pa), ga, _p(rsA), M, K, _p(W), ldw, _p(pw), n_blocks,
                             _p(csW), N, _p(bias), _p(Y), N if out is None else out.stride(0), _p(acc),
                             _stream(stream)), "qnn_qmatmul")
    return Y, acc


def _bad(what: str, *more):
    """Raises; messages are put together only here (a formatted type alone costs a microsecond)."""
    raise ValueError(what + "".join(f" {tuple(m) if isinstance(m, (tuple, list)) else m}" for m in more))


def _dtype(t, what: str) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        _bad(f"{what}: fp32, bf16 or fp16")
    return d


def _rows(t, what: str, dtype, shape) -> int:
    """Leading dimension of a matrix whose rows are contiguous."""
    if t.dtype is not dtype or t.shape != shape:
        _bad(what + ":", dtype, shape)
    s0, s1 = t.stride()
    cols = shape[1]
    if (s1 != 1 and cols > 1) or (s0 < cols and shape[0] > 1):
        _bad(what + ": rows of contiguous values, apart")
    return s0 if s0 >= cols else cols


def _flat(t, what: str, dtype, shape) -> int:
    """Address of a contiguous array, 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        _bad(what + ": contiguous", dtype, shape)
    return t.data_ptr()


def _frames(t, what: str, dtype, shape):
    """Address, sequence stride and frame stride of [B, T, ...] values whose frames are contiguous."""
    if t.dtype is not dtype or t.shape != shape:
        _bad(what + ":", dtype, shape)
    st = t.stride()
    if (st[-1] != 1 and shape[-1] > 1) or (len(st) == 4 and st[2] != shape[3] and shape[2] > 1):
        _bad(what + ": frames of contiguous values")
    return t.data_ptr(), st[0], st[1]


def _result(torch, shape, dtype, like, stream):
    """A new tensor for a call on stream, in memory of that stream: what the current one may still do with memory that was
    given back to it is not waited for there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _used(stream, *tensors):
    """Keeps the memory of a call's inputs from being given to others before what the call queued on stream is done."""
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


def qnn_rmsnorm_quantize(x, weight, residual=None, eps=1e-5, residual_out=None, want_values=False, stream=None):
    """Rows of x (+ residual) [rows, cols] (fp32, bf16 or fp16), through a root-mean-square norm with weight [cols] fp32, to
    8-bit codes, one unit per row. Returns (codes u8, params int32 [rows, 4], code_sums int32 [rows], h, values): h = x +
    residual in x's type (residual_out, which may be x or residual, or a new tensor; None without a residual), values the
    fp32 values that the codes stand for (None unless wanted). Rows of more than 8421504 values have no code_sums (None): they
    could pass 32 bits."""
    torch, L = _libs()
    if x.dim() != 2 or not x.is_cuda:
        _bad("x: a CUDA matrix")
    if stream is not None:
        _used(stream, x, weight, residual, residual_out)
        with torch.cuda.stream(stream):  # (the results are memory of the call's stream)
            return qnn_rmsnorm_quantize(x, weight, residual, eps, residual_out, want_values)
    shape, ty, dev, empty = x.shape, x.dtype, x.device, torch.empty
    dt = _dtype(x, "x")
    rows, cols = shape
    ldx = _rows(x, "x", ty, shape)
    h, pr, ph, ldr, ldh, pv = residual_out, 0, 0, 0, 0, 0
    if residual is not None:
        ldr = _rows(residual, "residual", ty, shape)
        pr = residual.data_ptr()
        if h is None:
            h, ldh = empty(shape, dtype=ty, device=dev), cols
        else:
            ldh = _rows(h, "residual_out", ty, shape)
        ph = h.data_ptr()
    elif h is not None:
        _bad("residual_out: needs a residual")
    w = _flat(weight, "weight", torch.float32, (cols,))
    codes = empty(shape, dtype=torch.uint8, device=dev)
    params = empty((rows, 4), dtype=torch.int32, device=dev)
    sums = empty((rows,), dtype=torch.int32, device=dev) if cols <= _MOST_SUMMED else None
    values = None
    if want_values:
        values = empty(shape, dtype=torch.float32, device=dev)
        pv = values.data_ptr()
    st = L.qnn_rmsnorm_quantize(x.data_ptr(), ldx, pr, ldr, dt, w, eps, rows, cols, ph, ldh, codes.data_ptr(), cols,
                                params.data_ptr(), sums.data_ptr() if sums is not None else 0, pv, cols, _here(torch))
    if st:
        _check(st, "qnn_rmsnorm_quantize")
    return codes, params, sums, h, values


class Weights4:
    """4-bit weights [N, K] with a scale and an offset per `group` columns of a row, as qnn_quantize4 lays them out: codes
    u8 [ceil(N/16), ceil(K/128), 1024], units bf16 [ceil(N/16), ceil(K/128), 16, 128 / group, 2] (offset, scale),
    row_sums fp32 [N]."""
    __slots__ = ("codes", "units", "row_sums", "N", "K", "group")

    def __init__(self, codes, units, row_sums, N: int, K: int, group: int):
        torch = _libs()[0]
        if group != 32 and group != 64 and group != 128:
            _bad("group: 32, 64 or 128")
        nt, kt = (N + 15) // 16, (K + 127) // 128
        _flat(codes, "codes", torch.uint8, (nt, kt, 1024))
        _flat(units, "units", torch.bfloat16, (nt, kt, 16, 128 // group, 2))
        _flat(row_sums, "row_sums", torch.float32, (N,))
        self.codes, self.units, self.row_sums, self.N, self.K, self.group = codes, units, row_sums, N, K, group


def qnn_quantize4(w, group: int = 64, stream=None) -> Weights4:
    """Weights w, CUDA fp32 [N, K], to 4-bit codes offline, one unit per group (32, 64 or 128) of a row's columns."""
    torch, L = _libs()
    if w.dim() != 2 or not w.is_cuda:
        _bad("w: a CUDA matrix")
    if group not in (32, 64, 128):
        _bad("group: 32, 64 or 128")
    N, K = w.shape
    ldw = _rows(w, "w", torch.float32, w.shape)
    tiles = ((N + 15) // 16, (K + 127) // 128)
    codes = _result(torch, (*tiles, 1024), torch.uint8, w, stream)
    units = _result(torch, (*tiles, 16, 128 // group, 2), torch.bfloat16, w, stream)
    sums = _result(torch, (N,), torch.float32, w, stream)
    if stream is not None:
        _used(stream, w)
    _check(L.qnn_quantize4(w.data_ptr(), N, K, ldw, group, codes.data_ptr(), units.data_ptr(), sums.data_ptr(),
                           _stream(stream)), "qnn_quantize4")
    return Weights4(codes, units, sums, N, K, group)


def qnn_qmatmul4(A, pa, weights: Weights4, ga=PER_ROW, bias=None, out=None, stream=None):
    """Y = R(A' W'^T) + bias with 4-bit weights: A u8 [M, K] codes with their units pa int32 [M, 4] (or [1, 4] with
    ga = PER_MATRIX), as qnn_quantize and qnn_rmsnorm_quantize give them. Returns Y fp32 [M, N]."""
    torch, L = _libs()
    if A.dim() != 2 or not A.is_cuda or A.shape[1] != weights.K:
        _bad("A: a CUDA matrix of the weights' K columns")
    M, K = shape = A.shape
    N = weights.N
    lda = _rows(A, "A", torch.uint8, shape)
    p = _flat(pa, "pa", torch.int32, (M if ga == PER_ROW else 1, 4))
    b = _flat(bias, "bias", torch.float32, (N,))
    if out is None:
        Y, ldy = _result(torch, (M, N), torch.float32, A, stream), N
    else:
        Y, ldy = out, _rows(out, "out", torch.float32, (M, N))
    if stream is not None:
        _used(stream, A, pa, weights.codes, weights.units, weights.row_sums, bias, out)
    st = L.qnn_qmatmul4(A.data_ptr(), lda, p, ga, M, K, weights.codes.data_ptr(), weights.units.data_ptr(), weights.group,
                        weights.row_sums.data_ptr(), N, b, Y.data_ptr(), ldy,
                        _here(torch) if stream is None else stream.cuda_stream)
    if st:
        _check(st, "qnn_qmatmul4")
    return Y


def qnn_causal_conv(x, weight, bias=None, silu=True, state_in=None, state_out=None, lengths=None, out=None, stream=None):
    """Short causal convolution over time of each channel, through SiLU unless silu is False: x [B, T, D] (fp32, bf16 or
    fp16; frames may be slices of wider ones), weight [D, W] and bias [D] fp32, states [B, W - 1, D] in x's type (state_out
    may be state_in), lengths int32 [B]. Returns out, [B, T, D]; without an out given, the frames behind a sequence's end
    hold nothing in particular."""
    torch, L = _libs()
    if x.dim() != 3 or not x.is_cuda:
        _bad("x: CUDA [B, T, D]")
    dt, ty = _dtype(x, "x"), x.dtype
    B, T, D = shape = x.shape
    if weight.dim() != 2:
        _bad("weight: [D, W]")
    W = weight.shape[1]
    y = out if out is not None else _result(torch, shape, ty, x, stream)
    px, xs, xf = _frames(x, "x", ty, shape)
    py, ys, yf = _frames(y, "out", ty, shape)
    state = (B, W - 1, D)
    if stream is not None:
        _used(stream, x, weight, bias, state_in, state_out, lengths, out)
    st = L.qnn_causal_conv(px, xs, xf, dt, B, T, D, _flat(weight, "weight", torch.float32, (D, W)), W,
                           _flat(bias, "bias", torch.float32, (D,)), 1 if silu else 0, _flat(state_in, "state_in", ty, state),
                           _flat(state_out, "state_out", ty, state), _flat(lengths, "lengths", torch.int32, (B,)), py, ys, yf,
                           _here(torch) if stream is None else stream.cuda_stream)
    if st:
        _check(st, "qnn_causal_conv")
    return y


def qnn_ssm_scan(u, dt, A, B, C, D=None, z=None, dt_bias=None, softplus=True, state_in=None, state_out=None, lengths=None,
                 out=None, stream=None):
    """Selective scan over time: u, dt and z [B, T, D] and B, C [B, T, groups, N] or [B, T, N] (fp32, bf16 or fp16, all of one
    type; frames may be slices of wider ones), A [D, N], D [D], dt_bias [D] and states [B, D, N] fp32 (state_out may be
    state_in), lengths int32 [B]. Returns out, [B, T, D]; without an out given, the frames behind a sequence's end hold
    nothing in particular."""
    torch, L = _libs()
    if u.dim() != 3 or not u.is_cuda:
        _bad("u: CUDA [B, T, D]")
    ty, f32, kind = u.dtype, torch.float32, _dtype(u, "u")
    nb, nt, nd = shape = u.shape
    if A.dim() != 2:
        _bad("A: [D, N]")
    ns = A.shape[1]
    groups, bc = 1, (nb, nt, ns)
    if B.dim() == 4:
        groups = B.shape[2]
        bc = (nb, nt, groups, ns)
    y = out if out is not None else _result(torch, shape, ty, u, stream)
    state = (nb, nd, ns)
    pz, zs, zf = _frames(z, "z", ty, shape) if z is not None else (0, 0, 0)
    args = _SSM_ARGS.pack(nb, nt, nd, ns, groups, kind, 1 if softplus else 0, *_frames(u, "u", ty, shape),
                          *_frames(dt, "dt", ty, shape), *_frames(B, "B", ty, bc), *_frames(C, "C", ty, bc), pz, zs, zf,
                          *_frames(y, "out", ty, shape), _flat(A, "A", f32, (nd, ns)), _flat(D, "D", f32, (nd,)),
                          _flat(dt_bias, "dt_bias", f32, (nd,)), _flat(state_in, "state_in", f32, state),
                          _flat(state_out, "state_out", f32, state), _flat(lengths, "lengths", torch.int32, (nb,)))
    if stream is not None:
        _used(stream, u, dt, A, B, C, D, z, dt_bias, state_in, state_out, lengths, out)
    st = L.qnn_ssm_scan(args, _here(torch) if stream is None else stream.cuda_stream)
    if st:
        _check(st, "qnn_ssm_scan")
    return y


def lstm_desc(num_layers, input_dim, hidden, proj=0, num_classes=0, output_mode=None, stack=0,
              stack_stride=0, weight_blocks=0) -> LstmDesc:
    if output_mode is None:
        output_mode = OUT_QUANT if num_classes > 0 else OUT_NONE
    return LstmDesc(num_layers, input_dim, hidden, proj, num_classes, output_mode, stack, stack_stride,
                    weight_blocks)


def stack_frames(x, n: int, stride: int, out=None, stream=None):
    """Sec. 4 frontend on a CUDA tensor x [B, T, I]: [B, ceil(T/stride), n*I], input t' = frames
    stride*t' .. stride*t' + n - 1 concatenated (the last frame standing in past the end)."""
    import torch
    B, T, I = x.shape
    if out is None:
        out = torch.empty((B, (T + stride - 1) // stride, n * I), dtype=torch.float32, device=x.device)
    _check(lib().qnn_stack_frames(_p(x), B, T, I, n, stride, _p(out), _stream(stream)), "qnn_stack_frames")
    return out


def qnn_lstm_param_count(d: LstmDesc) -> int:
    return int(lib().qnn_lstm_param_count(C.byref(d)))


class LstmModel:
    """Owns a qnn_lstm_model handle: weights quantized offline at construction (Sec. 3.1)."""

    def __init__(self, d: LstmDesc, params):
        self.desc = d
        self.R = d.proj if d.proj > 0 else d.hidden
        n = qnn_lstm_param_count(d)
        if n < 0:
            raise QnnError(QNN_ERR_INVALID_ARG, "qnn_lstm_param_count")
        assert int(params.numel() if hasattr(params, "numel") else params.size) == n
        h = C.c_void_p()
        _check(lib().qnn_lstm_model_create(C.byref(d), _p(params), C.byref(h)), "qnn_lstm_model_create")
        self._h = h

    def close(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.qnn_lstm_model_destroy(self._h)
            self._h = None

    __del__ = close

    def weights(self):
        """(codes u8 [param_count] in the packed layout, params records per unit)."""
        n = qnn_lstm_param_count(self.desc)
        codes = np.zeros(n, np.uint8)
        nu = C.c_int64(0)
        _check(lib().qnn_lstm_model_weights(self._h, None, None, C.byref(nu)), "qnn_lstm_model_weights")
        prm = np.zeros(nu.value, QPARAMS_DTYPE)
        _check(lib().qnn_lstm_model_weights(self._h, _p(codes), _p(prm), C.byref(nu)), "qnn_lstm_model_weights")
        return codes, prm

    def forward(self, x, y=None, h_state=None, c_state=None, h_all=None, stream=None, logits=None):
        """x [B, T, I] fp32 (CUDA tensor, or numpy/pinned CPU tensor: copied inside the call).
        Returns y ([B, T, C] or [B, T, R]). A y given in pinned CPU memory receives the posteriors
        from the softmax kernel directly; with any CPU buffer, synchronize the stream before
        reading it. logits: optional [B, T, C] buffer (host or device) that receives the output
        layer's values before the softmax (qnn_lstm_forward_logits)."""
        import torch
        B, T, I = x.shape
        d = self.desc
        ycols = d.num_classes if d.num_classes > 0 else self.R
        if d.stack_stride > 1:  # frame stacking: one network input every stack_stride frames
            T = (T + d.stack_stride - 1) // d.stack_stride
        if y is None:
            if isinstance(x, np.ndarray):
                y = np.empty((B, T, ycols), np.float32)
            else:
                y = torch.empty((B, T, ycols), dtype=torch.float32, device=x.device)
        if logits is None:
            _check(lib().qnn_lstm_forward(self._h, _p(x), B, x.shape[1], _p(y), _p(h_state), _p(c_state),
                                          _p(h_all), _stream(stream)), "qnn_lstm_forward")
        else:
            _check(lib().qnn_lstm_forward_logits(self._h, _p(x), B, x.shape[1], _p(y), _p(logits), _p(h_state),
                                                 _p(c_state), _p(h_all), _stream(stream)), "qnn_lstm_forward_logits")
        return y


class LstmStream:
    """Streaming server mode (qnn_lstm_stream_*): B sequences fed frame by frame to a resident
    kernel; push() appends frames [B, n, I], pull() returns the next frames' outputs [B, n, out]
    (posteriors, or top-layer outputs without an output layer). Host numpy arrays only."""

    def __init__(self, model: LstmModel, B: int, chunk: int = 1024, idle_seconds: float = 10.0):
        self.model, self.B = model, B
        d = model.desc
        self.I = d.input_dim * max(d.stack, 1)
        self.out_dim = d.num_classes if d.num_classes > 0 else model.R
        h = C.c_void_p()
        _check(lib().qnn_lstm_stream_open(model._h, B, chunk, idle_seconds, C.byref(h)), "qnn_lstm_stream_open")
        self._h = h

    def push(self, x: np.ndarray):
        x = np.ascontiguousarray(x, dtype=np.float32)
        assert x.ndim == 3 and x.shape[0] == self.B and x.shape[2] == self.I
        _check(lib().qnn_lstm_stream_push(self._h, _p(x), x.shape[1]), "qnn_lstm_stream_push")

    def pull(self, n: int, timeout: float = 10.0) -> np.ndarray:
        y = np.empty((self.B, n, self.out_dim), np.float32)
        _check(lib().qnn_lstm_stream_pull(self._h, _p(y), n, timeout), "qnn_lstm_stream_pull")
        return y

    def close(self) -> int:
        """Ends the session; returns the first status the kernel recorded (QNN_OK if none)."""
        st = QNN_OK
        if getattr(self, "_h", None) and _lib is not None:
            st = _lib.qnn_lstm_stream_close(self._h)
            self._h = None
        return st

    __del__ = close

"""Python binding of libmxq (include/mxq.h): argument marshalling only.

Every step of the quantize / pack / GEMM path runs in the HIP kernels of
``libmxq.so``; torch provides device memory and the current stream.  There
is no fallback: if the library is missing the calls raise ``MxqError``.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmxq.so")
BLOCK = 32
DECODE_MAX_M = 64


class MxqError(RuntimeError):
    pass


class _Fmt(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int64), ("block", ctypes.c_int32),
                ("round", ctypes.c_int32), ("clamp", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("widths", ctypes.c_void_p),
                ("perm", ctypes.c_void_p)]


class _Rotary(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("positions", ctypes.c_int64),
                ("rot", ctypes.c_int32), ("layout", ctypes.c_int32)]


class _PagedKv(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int64), ("Hkv", ctypes.c_int64),
                ("page_tokens", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("k_mant", ctypes.c_void_p), ("k_exp", ctypes.c_void_p),
                ("v_mant", ctypes.c_void_p), ("v_exp", ctypes.c_void_p)]


class _PagedBatch(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int64), ("T", ctypes.c_int64), ("max_q", ctypes.c_int64),
                ("max_kv", ctypes.c_int64), ("cu_q", ctypes.c_void_p),
                ("kv_len", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("ld_table", ctypes.c_int64), ("table_pages", ctypes.c_int64)]


class _AttnOpts(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("softcap", ctypes.c_float),
                ("window", ctypes.c_int64), ("prefix", ctypes.c_void_p),
                ("slopes", ctypes.c_void_p)]


class _Experts(ctypes.Structure):
    _fields_ = [("pairs", ctypes.c_int64), ("experts", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("first", ctypes.c_void_p),
                ("pair", ctypes.c_void_p), ("work", ctypes.c_void_p)]


class _RouteOpts(ctypes.Structure):
    _fields_ = [("k", ctypes.c_int32), ("score", ctypes.c_int32), ("normalise", ctypes.c_int32),
                ("scale", ctypes.c_float), ("bias", ctypes.c_void_p)]


class _QkNorm(ctypes.Structure):
    _fields_ = [("q_gain", ctypes.c_void_p), ("k_gain", ctypes.c_void_p), ("eps", ctypes.c_float)]


EXPERT_WORK = 64
_SCORES = {"softmax": 0, "sigmoid": 1}

_lib = None

# name -> (restype, argtypes)
_P, _I64 = ctypes.c_void_p, ctypes.c_int64
_SIGS = {
    "mxq_abi_version": (ctypes.c_int, []),
    "mxq_status_str": (ctypes.c_char_p, [ctypes.c_int]),
    "mxq_act_packed_bytes": (_I64, [_P]),
    "mxq_exp_row_bytes": (_I64, [_P]),
    "mxq_act_bytes": (_I64, [_P, _I64]),
    "mxq_act_exp_bytes": (_I64, [_P, _I64]),
    "mxq_weight_bytes": (_I64, [_P, _I64]),
    "mxq_weight_exp_bytes": (_I64, [_P, _I64]),
    "mxq_quantize_act": (ctypes.c_int, [_P, _P, _I64, _I64, _P, _P, _P]),
    "mxq_quantize_rows": (ctypes.c_int, [_P, _P, _I64, _I64, _P, _P, _P]),
    "mxq_quantize_act_rmsnorm": (ctypes.c_int, [_P, _P, _I64, _I64, _P, ctypes.c_float,
                                                 _P, _P, _P]),
    "mxq_quantize_act_swiglu": (ctypes.c_int, [_P, _P, _P, _I64, _I64, _P, _P, _P]),
    "mxq_pack_weights": (ctypes.c_int, [_P, _P, _I64, _I64, _P, _P, _P]),
    "mxq_gemm": (ctypes.c_int, [_P, _I64, _I64, _P, _P, _P, _P, _P, _I64, _P]),
    "mxq_gemm_partials": (ctypes.c_int, [_P, _I64, _I64, _P, _P, _P, _P, _P, _P]),
    "mxq_unpack_act": (ctypes.c_int, [_P, _I64, _P, _P, _P, _P, _P]),
    "mxq_unpack_weights": (ctypes.c_int, [_P, _I64, _P, _P, _P, _P, _P]),
    "mxq_calib_colsq": (ctypes.c_int, [_P, _I64, _I64, _I64, _P, ctypes.c_int, _P]),
    "mxq_calib_colsq_samples": (ctypes.c_int, [_P, _I64, _I64, _I64, _I64, _I64, _P, _P,
                                               ctypes.c_int, _P]),
    "mxq_calib_colsq_list": (ctypes.c_int, [_P, _P, _P, _I64, _I64, _P, _P, ctypes.c_int, _P]),
    "mxq_calib_ratio": (ctypes.c_int, [ctypes.c_int32, _P, _P, ctypes.c_double, _P]),
    "mxq_calib_counts": (ctypes.c_int, [_I64, ctypes.c_double, ctypes.c_double,
                                        ctypes.c_int32, _P, _P, _P]),
    "mxq_calib_perm": (ctypes.c_int, [_P, _I64, ctypes.c_int32, ctypes.c_int32, _P, _P]),
    "mxq_peak_sink_words": (_I64, []),
    "mxq_peak_stream_read": (ctypes.c_int, [_P, _I64, _P, _P]),
    "mxq_peak_mfma": (ctypes.c_int, [ctypes.c_int, _I64, _P, _P, _P]),
    "mxq_attn_work_bytes": (_I64, [_P, _I64, _I64, _I64, _I64]),
    "mxq_attn_decode": (ctypes.c_int, [_P, _P, _I64, _I64, _I64, _I64, ctypes.c_float,
                                       _P, _P, _P, _P, _P, _P, _I64, _P]),
    "mxq_attn_decode_static": (ctypes.c_int, [_P, _P, _I64, _I64, _I64, _I64, ctypes.c_float,
                                              _P, _P, _P, _P, _P, _P]),
    "mxq_rope_table": (ctypes.c_int, [_P, ctypes.c_int32, _I64, ctypes.c_double, _P, _P]),
    "mxq_rope": (ctypes.c_int, [_P, _P, _I64, _I64, _I64, _I64, _I64, _P, _P, _I64, _I64, _P]),
    "mxq_kv_page_bytes": (_I64, [_P, _I64, ctypes.c_int32]),
    "mxq_kv_page_exp_bytes": (_I64, [_P, _I64, ctypes.c_int32]),
    "mxq_kv_append": (ctypes.c_int, [_P, _P, _P, _I64, _I64, _P, _I64, _I64, _I64, _P, _P, _P,
                                     _P, _I64, _I64, _I64, _P, _P]),
    "mxq_kv_read": (ctypes.c_int, [_P, _P, _P, _I64, _P, _P, _P]),
    "mxq_attn_paged_work_bytes": (_I64, [_P, _P, _I64, _I64, _I64, _I64, _I64]),
    "mxq_attn_paged": (ctypes.c_int, [_P, _P, _P, _P, _P, _I64, _I64, _I64, _P, ctypes.c_int,
                                      _P, _I64, _P]),
    "mxq_expert_rows": (_I64, [_I64, ctypes.c_int32]),
    "mxq_route": (ctypes.c_int, [_P, _P, ctypes.c_int, _I64, _I64, _P, _P, _P, _P]),
    "mxq_expert_plan": (ctypes.c_int, [_P, _P, _P]),
    "mxq_quantize_act_experts": (ctypes.c_int, [_P, _P, _P, _P, _I64, _I64, _P, _P, _P]),
    "mxq_quantize_act_swiglu_experts": (ctypes.c_int, [_P, _P, _P, _P, _P, _I64, _I64, _P, _P,
                                                       _P]),
    "mxq_gemm_experts": (ctypes.c_int, [_P, _P, _I64, _P, _P, _P, _P, _P, ctypes.c_int, _I64, _P]),
    "mxq_combine_experts": (ctypes.c_int, [_P, ctypes.c_int, _I64, _P, _P, _I64, _I64,
                                           ctypes.c_int32, _I64, _P, _I64, _P, ctypes.c_int, _I64,
                                           _P]),
    "mxq_rope_qk": (ctypes.c_int, [_P, _P, _P, _I64, _I64] + [_P, _I64, _I64, _I64, _P, _I64,
                                                              _I64] * 2 + [_P]),
    "mxq_kv_append_norm": (ctypes.c_int, [_P, _P, _P, _P, _I64, _I64, _P, _I64, _I64, _I64, _P, _P,
                                          _P, _P, _I64, _I64, _I64, _P, _P]),
}


def lib(path: str = LIB_PATH):
    """Load libmxq.so (once).  Raises MxqError if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(path):
            raise MxqError("libmxq.so is not built (%s); run __graft_entry__.build()"
                           % path)
        handle = ctypes.CDLL(path)
        for name, (res, args) in _SIGS.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def _check(status: int, what: str):
    if status != 0:
        msg = lib().mxq_status_str(status).decode()
        raise MxqError("%s failed: %s (status %d)" % (what, msg, status))


def _size(v: int, what: str) -> int:
    if v < 0:
        _check(int(-v), what)
    return int(v)


def _stream():
    """The current stream's handle (of the current device, as
    torch.cuda.current_stream(), without the 3 us of its Stream object)."""
    if torch.cuda.is_initialized():
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream


def _ptr(t):
    return None if t is None else t.data_ptr()


class Format:
    """Width map + permutation of one quantized linear (include/mxq.h mxq_fmt).

    widths: K/32 entries in {3, 4, 6, 8}, non-decreasing (3-bit blocks are
            the floor of the 3-6-8 template).
    perm:   None (identity) or an int32 device tensor of K source columns.
    """

    def __init__(self, K: int, widths, perm=None, round: str = "rne",
                 clamp: str = "sym"):
        self.K = int(K)
        self.widths = np.ascontiguousarray(np.asarray(widths, dtype=np.uint8))
        if perm is not None:
            if not (isinstance(perm, torch.Tensor) and perm.is_cuda
                    and perm.dtype == torch.int32 and perm.is_contiguous()):
                raise MxqError("perm must be a contiguous int32 device tensor")
        self.perm = perm
        self.round = {"rne": 0, "rna": 1}[round]
        self.clamp = {"sym": 0, "full": 1}[clamp]
        self._c = _Fmt(self.K, BLOCK, self.round, self.clamp, 0,
                       self.widths.ctypes.data_as(ctypes.c_void_p).value,
                       None if perm is None else perm.data_ptr())
        self._ref = ctypes.byref(self._c)
        self._of = None
        self._unit = None

    @property
    def ref(self):
        return self._ref

    def _units(self):
        """What every size is a multiple of: the bytes of a 16-row activation
        tile and its scales, a 128-column weight super-slab and its scales, a
        packed row, an exponent row.  Asked of the library once per width map:
        a serving loop checks its buffers on every call.  (The shift that counts
        the tiles refuses a fraction.)"""
        w = self.widths.tobytes()
        if w != self._of:
            L, r = lib(), self._ref
            self._unit = tuple(_size(v, name) for v, name in (
                (L.mxq_act_bytes(r, 1), "mxq_act_bytes"),
                (L.mxq_act_exp_bytes(r, 1), "mxq_act_exp_bytes"),
                (L.mxq_weight_bytes(r, 1), "mxq_weight_bytes"),
                (L.mxq_weight_exp_bytes(r, 1), "mxq_weight_exp_bytes"),
                (L.mxq_act_packed_bytes(r), "mxq_act_packed_bytes"),
                (L.mxq_exp_row_bytes(r), "mxq_exp_row_bytes")))
            self._of = w
        return self._unit

    @property
    def nb(self) -> int:
        return self.K // BLOCK

    def act_packed_bytes(self) -> int:
        """Bytes of one packed activation row."""
        return self._units()[4]

    def exp_row_bytes(self) -> int:
        """Bytes of one row of block exponents."""
        return self._units()[5]

    def act_bytes(self, M: int) -> int:
        """The activation operand image of M rows (mxq_quantize_act)."""
        if M < 0:
            _check(2, "mxq_act_bytes")
        return (M + 15 >> 4) * self._units()[0]

    def act_exp_bytes(self, M: int) -> int:
        """Its scale bytes."""
        if M < 0:
            _check(2, "mxq_act_exp_bytes")
        return (M + 15 >> 4) * self._units()[1]

    def weight_bytes(self, N: int) -> int:
        if N < 0:
            _check(2, "mxq_weight_bytes")
        return (N + 127 >> 7) * self._units()[2]

    def weight_exp_bytes(self, N: int) -> int:
        if N < 0:
            _check(2, "mxq_weight_exp_bytes")
        return (N + 127 >> 7) * self._units()[3]


def _bf16_2d(t, K, what):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == torch.bfloat16
            and t.dim() == 2 and t.stride(1) == 1):
        raise MxqError("%s must be a 2-D bf16 device tensor with unit column stride"
                       % what)
    if t.shape[1] < K:
        raise MxqError("%s has fewer than K columns" % what)
    return t


def _dev_bytes(t, n: int, what: str, dev=None):
    """A contiguous uint8 device tensor of at least n bytes (on `dev`)."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is torch.uint8
            and t.is_contiguous()):
        raise MxqError("%s must be a contiguous uint8 device tensor" % what)
    if t.numel() < n:
        raise MxqError("%s holds %d bytes, %d needed" % (what, t.numel(), n))
    if dev is not None and t.device != dev:
        raise MxqError("%s is on %s, not %s" % (what, t.device, dev))
    return t


def _act_out(out, fmt: Format, M: int, dev):
    """The caller's (mant, exp) activation buffers, checked, or new ones."""
    if out is None:
        return (torch.empty(fmt.act_bytes(M), dtype=torch.uint8, device=dev),
                torch.empty(fmt.act_exp_bytes(M), dtype=torch.uint8, device=dev))
    mant, exp = out
    _dev_bytes(mant, fmt.act_bytes(M), "activation mantissa buffer", dev)
    _dev_bytes(exp, fmt.act_exp_bytes(M), "activation exponent buffer", dev)
    return mant, exp


def _gemm_operands(a_mant, a_exp, w_mant, w_exp, fmt: Format, M: int, N: int):
    if M < 0 or N < 0:
        raise MxqError("M and N must be non-negative")
    dev = a_mant.device if isinstance(a_mant, torch.Tensor) else None
    _dev_bytes(a_mant, fmt.act_bytes(M), "a_mant", dev)
    _dev_bytes(a_exp, fmt.act_exp_bytes(M), "a_exp", dev)
    _dev_bytes(w_mant, fmt.weight_bytes(N), "w_mant", dev)
    _dev_bytes(w_exp, fmt.weight_exp_bytes(N), "w_exp", dev)
    return dev


def quantize_act(a, fmt: Format, out=None):
    """Online activation quantization: bf16 [M, >=K] -> (mant uint8
    [act_bytes(M)], exp uint8 [act_exp_bytes(M)]) on the current stream."""
    _bf16_2d(a, fmt.K, "activations")
    M = a.shape[0]
    mant, exp = _act_out(out, fmt, M, a.device)
    _check(lib().mxq_quantize_act(fmt.ref, _ptr(a), M, a.stride(0), _ptr(mant),
                                  _ptr(exp), _stream()), "mxq_quantize_act")
    return mant, exp


def quantize_act_rmsnorm(x, gain, eps: float, fmt: Format, out=None):
    """RMS-normalise bf16 rows x with bf16 gain, then quantize them (one
    kernel; the normalised rows are never written)."""
    _bf16_2d(x, fmt.K, "activations")
    if gain.dtype != torch.bfloat16 or gain.numel() < fmt.K or not gain.is_contiguous():
        raise MxqError("gain must be a contiguous bf16 tensor of K elements")
    if not gain.is_cuda or gain.device != x.device:
        raise MxqError("gain must be on the activations' device")
    M = x.shape[0]
    mant, exp = _act_out(out, fmt, M, x.device)
    _check(lib().mxq_quantize_act_rmsnorm(fmt.ref, _ptr(x), M, x.stride(0), _ptr(gain),
                                          float(eps), _ptr(mant), _ptr(exp), _stream()),
           "mxq_quantize_act_rmsnorm")
    return mant, exp


def quantize_act_swiglu(gate, up, fmt: Format, out=None):
    """Quantize SiLU(gate) * up (bf16 rows of the same shape and stride) in
    one kernel; the product rows are never written."""
    _bf16_2d(gate, fmt.K, "gate")
    _bf16_2d(up, fmt.K, "up")
    if up.shape != gate.shape or up.stride() != gate.stride():
        raise MxqError("gate and up must have the same shape and strides")
    if up.device != gate.device:
        raise MxqError("gate and up must be on one device")
    M = gate.shape[0]
    mant, exp = _act_out(out, fmt, M, gate.device)
    _check(lib().mxq_quantize_act_swiglu(fmt.ref, _ptr(gate), _ptr(up), M, gate.stride(0),
                                         _ptr(mant), _ptr(exp), _stream()),
           "mxq_quantize_act_swiglu")
    return mant, exp


def quantize_rows(a, fmt: Format, out=None):
    """The quantizer writing packed rows: bf16 [M, >=K] -> (rows uint8
    [M, act_packed_bytes], exps uint8 [M, exp_row_bytes]) -- the KV-cache
    layout, and the input of unpack_act and gemm_partials."""
    _bf16_2d(a, fmt.K, "activations")
    M = a.shape[0]
    rb, erb = fmt.act_packed_bytes(), fmt.exp_row_bytes()
    if out is None:
        rows = torch.empty((M, rb), dtype=torch.uint8, device=a.device)
        exps = torch.empty((M, erb), dtype=torch.uint8, device=a.device)
    else:
        rows, exps = out
        _dev_bytes(rows, M * rb, "packed row buffer", a.device)
        _dev_bytes(exps, M * erb, "exponent row buffer", a.device)
    _check(lib().mxq_quantize_rows(fmt.ref, _ptr(a), M, a.stride(0), _ptr(rows),
                                   _ptr(exps), _stream()), "mxq_quantize_rows")
    return rows, exps


def pack_weights(w, fmt: Format):
    """Offline weight quantization into the GEMM-tiled packed layout."""
    _bf16_2d(w, fmt.K, "weights")
    N = w.shape[0]
    mant = torch.empty(fmt.weight_bytes(N), dtype=torch.uint8, device=w.device)
    exp = torch.empty(fmt.weight_exp_bytes(N), dtype=torch.uint8, device=w.device)
    _check(lib().mxq_pack_weights(fmt.ref, _ptr(w), N, w.stride(0), _ptr(mant),
                                  _ptr(exp), _stream()), "mxq_pack_weights")
    return mant, exp


def gemm(a_mant, a_exp, w_mant, w_exp, fmt: Format, M: int, N: int, out=None):
    """Y = Ahat @ What^T, fp32 [M, N]."""
    dev = _gemm_operands(a_mant, a_exp, w_mant, w_exp, fmt, M, N)
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=dev)
    if not (isinstance(out, torch.Tensor) and out.is_cuda and out.device == dev
            and out.dim() == 2 and out.stride(1) == 1 and out.dtype == torch.float32):
        raise MxqError("out must be a 2-D fp32 device tensor with unit column stride")
    if out.shape[0] < M or out.shape[1] < N:
        raise MxqError("out is %s, smaller than [M, N] = [%d, %d]" % (tuple(out.shape), M, N))
    _check(lib().mxq_gemm(fmt.ref, M, N, _ptr(a_mant), _ptr(a_exp), _ptr(w_mant),
                          _ptr(w_exp), _ptr(out), out.stride(0), _stream()),
           "mxq_gemm")
    return out


def gemm_partials(rows, exps, w_mant, w_exp, fmt: Format, M: int, N: int):
    """Exact per-block int32 sums P[M, N, K/32] (debug / parity) from packed
    rows (quantize_rows) and the packed weights."""
    if M < 0 or N < 0:
        raise MxqError("M and N must be non-negative")
    dev = rows.device if isinstance(rows, torch.Tensor) else None
    _dev_bytes(rows, M * fmt.act_packed_bytes(), "rows", dev)
    _dev_bytes(exps, M * fmt.exp_row_bytes(), "exps", dev)
    _dev_bytes(w_mant, fmt.weight_bytes(N), "w_mant", dev)
    _dev_bytes(w_exp, fmt.weight_exp_bytes(N), "w_exp", dev)
    a_mant, a_exp = rows, exps
    p = torch.empty((M, N, fmt.nb), dtype=torch.int32, device=dev)
    _check(lib().mxq_gemm_partials(fmt.ref, M, N, _ptr(a_mant), _ptr(a_exp),
                                   _ptr(w_mant), _ptr(w_exp), _ptr(p), _stream()),
           "mxq_gemm_partials")
    return p


def unpack_act(mant, exp, fmt: Format, rows: int):
    """Packed rows and exponent rows (quantize_rows) -> (q int8 [rows, K],
    e uint8 [rows, K/32])."""
    _dev_bytes(mant, rows * fmt.act_packed_bytes(), "rows")
    _dev_bytes(exp, rows * fmt.exp_row_bytes(), "exps", mant.device)
    q = torch.empty((rows, fmt.K), dtype=torch.int8, device=mant.device)
    e = torch.empty((rows, fmt.nb), dtype=torch.uint8, device=mant.device)
    _check(lib().mxq_unpack_act(fmt.ref, rows, _ptr(mant), _ptr(exp), _ptr(q), _ptr(e),
                                _stream()), "mxq_unpack_act")
    return q, e


def unpack_weights(w_mant, w_exp, fmt: Format, N: int):
    _dev_bytes(w_mant, fmt.weight_bytes(N), "w_mant")
    _dev_bytes(w_exp, fmt.weight_exp_bytes(N), "w_exp", w_mant.device)
    q = torch.empty((N, fmt.K), dtype=torch.int8, device=w_mant.device)
    e = torch.empty((N, fmt.nb), dtype=torch.uint8, device=w_mant.device)
    _check(lib().mxq_unpack_weights(fmt.ref, N, _ptr(w_mant), _ptr(w_exp), _ptr(q),
                                    _ptr(e), _stream()), "mxq_unpack_weights")
    return q, e


# --------------------------------------------------------------------------
# Achievable-peak microbenchmarks (measurement only)

def peak_sink(device):
    """A sink buffer large enough for the peak microbenchmarks."""
    return torch.empty(int(lib().mxq_peak_sink_words()), dtype=torch.int32, device=device)


def peak_stream_read(buf, sink):
    """Read every byte of `buf` (a device tensor, nbytes % 16 == 0) once."""
    nbytes = buf.numel() * buf.element_size()
    _check(lib().mxq_peak_stream_read(_ptr(buf), nbytes, _ptr(sink), _stream()),
           "mxq_peak_stream_read")
    return nbytes


PEAK_KINDS = {"int8": 0, "fp6": 1, "fp8": 2}


def peak_mfma(kind: str, iters: int, sink):
    """Matrix-core loop of `kind` ("int8", "fp6", "fp8"); returns the ops of
    one launch."""
    ops = ctypes.c_int64(0)
    _check(lib().mxq_peak_mfma(PEAK_KINDS[kind], int(iters), _ptr(sink),
                               ctypes.byref(ops), _stream()), "mxq_peak_mfma")
    return ops.value


# --------------------------------------------------------------------------
# Calibration (offline): permutation and width map from calibration samples

def _sample(x, dim: int):
    """A calibration sample (or, 3-D, a batch of them), checked."""
    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dtype == torch.bfloat16
            and x.dim() == dim and x.stride(dim - 1) == 1):
        raise MxqError("calibration samples must be %d-D bf16 device tensors with unit "
                       "column stride" % dim)
    return x


def _dev_array(t, n: int, dtype, what: str, dev):
    """A contiguous device array of at least n elements on `dev`."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype
            and t.is_contiguous()):
        raise MxqError("%s must be a contiguous %s device tensor" % (what, dtype))
    if t.numel() < n:
        raise MxqError("%s holds %d elements, %d needed" % (what, t.numel(), n))
    if t.device != dev:
        raise MxqError("%s is on %s, not %s" % (what, t.device, dev))
    return t


def calib_colsq(x, s=None, accumulate: bool = False):
    """Column sensitivities of one calibration sample x (bf16 [rows, K]):
    s[k] = sum_r x[r, k]^2 in float64 (added to s when accumulate).  s holds
    at least K columns; those past K stay as they are."""
    rows, K = _sample(x, 2).shape
    if s is None:
        if accumulate:
            raise MxqError("accumulate needs the running sensitivities")
        s = torch.empty(K, dtype=torch.float64, device=x.device)
    _dev_array(s, K, torch.float64, "sensitivities", x.device)
    _check(lib().mxq_calib_colsq(_ptr(x), rows, x.stride(0), K, _ptr(s),
                                 1 if accumulate else 0, _stream()), "mxq_calib_colsq")
    return s


def calib_colsq_samples(x, s=None, accumulate: bool = False, work=None):
    """Column sensitivities of a batch of samples x (bf16 [n, rows, K]),
    summed in sample order (equal to one calib_colsq call per sample)."""
    n, rows, K = _sample(x, 3).shape
    if s is None:
        if accumulate:
            raise MxqError("accumulate needs the running sensitivities")
        s = torch.empty(K, dtype=torch.float64, device=x.device)
    if work is None:
        work = torch.empty(n * K, dtype=torch.float64, device=x.device)
    _dev_array(s, K, torch.float64, "sensitivities", x.device)
    _dev_array(work, n * K, torch.float64, "work", x.device)
    _check(lib().mxq_calib_colsq_samples(_ptr(x), n, rows, x.stride(1), x.stride(0), K,
                                         _ptr(work), _ptr(s), 1 if accumulate else 0,
                                         _stream()), "mxq_calib_colsq_samples")
    return s


def calib_ratio(d_in, s_layer, B: float) -> float:
    """Theorem A.1's control parameter R for layers of widths d_in."""
    n = len(d_in)
    d = (ctypes.c_int64 * n)(*[int(v) for v in d_in])
    sl = (ctypes.c_double * n)(*[float(v) for v in s_layer])
    R = ctypes.c_double(0.0)
    _check(lib().mxq_calib_ratio(n, d, sl, float(B), ctypes.byref(R)), "mxq_calib_ratio")
    return R.value


def calib_counts(d_in: int, R: float, s_layer: float, n8_blocks: int = 1):
    """(n4, n6, n8) block counts of one layer (Algorithm 2)."""
    out = [ctypes.c_int32(0) for _ in range(3)]
    _check(lib().mxq_calib_counts(int(d_in), float(R), float(s_layer), int(n8_blocks),
                                  *[ctypes.byref(v) for v in out]), "mxq_calib_counts")
    return tuple(v.value for v in out)


def calib_perm(s, n6: int, n8: int, perm=None):
    """The permutation of Algorithm 2 (int32 device tensor [K])."""
    if not (isinstance(s, torch.Tensor) and s.is_cuda and s.dtype == torch.float64
            and s.dim() == 1 and s.is_contiguous()):
        raise MxqError("sensitivities must be a contiguous 1-D float64 device tensor")
    K = s.numel()
    if perm is None:
        perm = torch.empty(K, dtype=torch.int32, device=s.device)
    _dev_array(perm, K, torch.int32, "perm", s.device)
    _check(lib().mxq_calib_perm(_ptr(s), K, int(n6), int(n8), _ptr(perm), _stream()),
           "mxq_calib_perm")
    return perm


CALIB_LIST_MAX = 32


def _colsq_list(samples):
    """Sensitivities of samples that lie on the device together, a launch per
    CALIB_LIST_MAX samples: one sample's columns fill a fraction of the GPU.
    None for samples that are not all bf16 [rows, K] of one K and device
    (they are summed one call each)."""
    first = samples[0] if len(samples) > 1 else None
    if not (isinstance(first, torch.Tensor) and first.is_cuda and first.dim() == 2):
        return None
    K, dev = first.shape[1], first.device
    if not all(isinstance(x, torch.Tensor) and x.dim() == 2 and x.dtype is torch.bfloat16
               and x.stride(1) == 1 and x.shape[1] == K and x.device == dev for x in samples):
        return None
    s = torch.empty(K, dtype=torch.float64, device=dev)
    work = torch.empty(min(len(samples), CALIB_LIST_MAX) * K, dtype=torch.float64, device=dev)
    for i in range(0, len(samples), CALIB_LIST_MAX):
        part = samples[i:i + CALIB_LIST_MAX]
        n = len(part)
        _check(lib().mxq_calib_colsq_list((_P * n)(*[x.data_ptr() for x in part]),
                                          (_I64 * n)(*[x.shape[0] for x in part]),
                                          (_I64 * n)(*[x.stride(0) for x in part]), n, K,
                                          _ptr(work), _ptr(s), 1 if i else 0, _stream()),
               "mxq_calib_colsq_list")
    return s


def calibrate(samples, s_layer: float, R: float, n8_blocks: int = 1):
    """One layer: sensitivities over the samples, the block counts and the
    permutation.  Returns (perm int32 device tensor, widths list).  The first
    sample's width is the layer's: no later one may be wider (a narrower one
    counts for the columns that it has)."""
    s = _colsq_list(samples) if isinstance(samples, (list, tuple)) else None
    if s is None:
        if isinstance(samples, (list, tuple)):
            for x in samples:
                if _sample(x, 2).shape[1] > samples[0].shape[1]:
                    raise MxqError("a calibration sample is wider than the first one")
        for i, x in enumerate(samples):
            s = calib_colsq(x, s, accumulate=i > 0)
    K = s.numel()
    n4, n6, n8 = calib_counts(K, R, s_layer, n8_blocks)
    perm = calib_perm(s, n6, n8)
    return perm, [4] * n4 + [6] * n6 + [8] * n8


def attn_work_bytes(fmt: Format, B: int, Hq: int, Hkv: int, T: int) -> int:
    """Bytes of the scratch that mxq_attn_decode needs for these sizes."""
    return _size(lib().mxq_attn_work_bytes(fmt.ref, B, Hq, Hkv, T), "mxq_attn_work_bytes")


def attn_decode(q, k_cache, v_cache, fmt: Format, B: int, Hq: int, Hkv: int, T: int,
                scale: float, out=None, work=None):
    """Decode attention over an MXINT KV cache.  q: bf16 [B, Hq, 128] on the
    device; k_cache, v_cache: (rows, exps) as returned by quantize_rows for
    the B * T * Hkv cache rows (row (b * T + t) * Hkv + h).  Returns float32
    [B, Hq, 128] on the current stream."""
    if not (isinstance(q, torch.Tensor) and q.is_cuda and q.dtype == torch.bfloat16
            and q.is_contiguous() and q.numel() == B * Hq * 128):
        raise MxqError("q must be a contiguous bf16 device tensor of B * Hq * 128 elements")
    rows = B * T * Hkv
    for mant, exp in (k_cache, v_cache):
        if mant.numel() < rows * fmt.act_packed_bytes() or exp.numel() < rows * fmt.exp_row_bytes():
            raise MxqError("KV cache buffers are too small for B * T * Hkv rows")
    if out is None:
        out = torch.empty((B, Hq, 128), dtype=torch.float32, device=q.device)
    nw = attn_work_bytes(fmt, B, Hq, Hkv, T)
    if work is None:
        work = torch.empty(max(nw, 16), dtype=torch.uint8, device=q.device)
    _check(lib().mxq_attn_decode(fmt.ref, _ptr(q), B, Hq, Hkv, T, float(scale),
                                 _ptr(k_cache[0]), _ptr(k_cache[1]), _ptr(v_cache[0]),
                                 _ptr(v_cache[1]), _ptr(out), _ptr(work), work.numel(),
                                 _stream()), "mxq_attn_decode")
    return out


ATTN_STATIC_WORK_BYTES = 8 << 20


def attn_decode_static(q, k_cache, v_cache, fmt: Format, B: int, Hq: int, Hkv: int, T: int,
                       scale: float, out):
    """attn_decode without a work buffer: the library's static per-GPU
    scratch holds the split results (calls overlapping on one GPU race).
    `out` (float32 [B, Hq, 128], contiguous, on the device) is required, so
    the call allocates nothing."""
    if not (isinstance(q, torch.Tensor) and q.is_cuda and q.dtype == torch.bfloat16
            and q.is_contiguous() and q.numel() == B * Hq * 128):
        raise MxqError("q must be a contiguous bf16 device tensor of B * Hq * 128 elements")
    if not (isinstance(out, torch.Tensor) and out.is_cuda and out.dtype == torch.float32
            and out.is_contiguous() and out.numel() >= B * Hq * 128):
        raise MxqError("out must be a contiguous float32 device tensor of B * Hq * 128 elements")
    rows = B * T * Hkv
    for mant, exp in (k_cache, v_cache):
        if mant.numel() < rows * fmt.act_packed_bytes() or exp.numel() < rows * fmt.exp_row_bytes():
            raise MxqError("KV cache buffers are too small for B * T * Hkv rows")
    _check(lib().mxq_attn_decode_static(fmt.ref, _ptr(q), B, Hq, Hkv, T, float(scale),
                                        _ptr(k_cache[0]), _ptr(k_cache[1]), _ptr(v_cache[0]),
                                        _ptr(v_cache[1]), _ptr(out), _stream()),
           "mxq_attn_decode_static")
    return out


# --------------------------------------------------------------------------
# Rotary positions, the paged KV cache, and attention over it

def _current(dev, what: str):
    """The calls run on the current device's current stream: its handle."""
    i = torch._C._cuda_getDevice()
    if dev.index != i:
        raise MxqError("%s is on %s, which is not the current device" % (what, dev))
    return torch._C._cuda_getCurrentRawStream(i)


def _heads(t, what: str, dev=None, heads=None, D=None):
    """bf16 rows [tokens, heads, D] with unit stride along D: their shape."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is torch.bfloat16
            and t.dim() == 3 and (t.stride(2) == 1 or t.shape[2] <= 1)):
        raise MxqError("%s must be a 3-D bf16 device tensor [tokens, heads, D] with unit "
                       "stride along D" % what)
    if dev is not None and t.device != dev:
        raise MxqError("%s is on %s, not %s" % (what, t.device, dev))
    s = t.shape
    if (heads is not None and s[1] != heads) or (D is not None and s[2] != D):
        raise MxqError("%s is %s, not [tokens, %s, %s]" % (what, tuple(s), heads, D))
    return s


def _index(t, n: int, dtype, what: str, dev):
    """A contiguous 1-D integer device tensor of n elements: its address."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.dim() == 1
            and t.is_contiguous()):
        raise MxqError("%s must be a contiguous 1-D %s device tensor" % (what, dtype))
    if t.numel() != n:
        raise MxqError("%s holds %d elements, not %d" % (what, t.numel(), n))
    if t.device != dev:
        raise MxqError("%s is on %s, not %s" % (what, t.device, dev))
    return t.data_ptr()


def rope_inv_freq(rot: int, base: float = 10000.0, scaling: str | None = None,
                  factor: float = 1.0, orig_positions: int = 0, low: float = 1.0,
                  high: float = 32.0):
    """The rotary frequencies of a head whose first `rot` values turn, for a
    context `factor` times as long as the `orig_positions` a model was trained
    on: (float64 array [rot / 2], factor for the cosines and sines).

    None     f_i = base^(-2 i / rot).
    "linear" f_i / factor: all positions squeezed into the trained range.
    "base"   base * factor^(rot / (rot - 2)): the lowest frequency is divided by
             the factor, the highest stays.
    "ramp"   by the turns r_i = orig_positions f_i / 2 pi that a frequency makes
             in the trained range: f_i for r_i >= high, f_i / factor for r_i <=
             low, between the two their mix, linear in i from the index that
             makes `high` turns (rounded down, at least 0) to the one that makes
             `low` (rounded up, also where it lies past the last frequency);
             cosines and sines are scaled by 1 + 0.1 ln(factor).
    "bands"  the mix linear in r_i instead, and cosines and sines as they are.
    """
    if rot < 2 or rot % 2:
        raise MxqError("rot must be even and at least 2")
    if not (np.isfinite(base) and base > 0 and np.isfinite(factor) and factor >= 1):
        raise MxqError("base must be positive and factor at least 1")
    i = np.arange(rot // 2, dtype=np.float64)
    f = float(base) ** (-2.0 * i / rot)
    if scaling is None:
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "base":
        if rot == 2:                       # one frequency, which is 1
            return f, 1.0
        return (base * factor ** (rot / (rot - 2.0))) ** (-2.0 * i / rot), 1.0
    if scaling not in ("ramp", "bands"):
        raise MxqError("scaling must be None, 'linear', 'base', 'ramp' or 'bands'")
    if not (1 <= orig_positions < np.inf and 0 < low < high < np.inf):
        raise MxqError("%r needs orig_positions and 0 < low < high" % scaling)
    turns = orig_positions * f / (2 * np.pi)
    if scaling == "bands":
        keep = np.clip((turns - low) / (high - low), 0.0, 1.0)
        return keep * f + (1 - keep) * f / factor, 1.0
    if base <= 1.0:                        # (frequencies that do not fall)
        raise MxqError("'ramp' needs a base above 1")

    def index(t):
        return rot * np.log(orig_positions / (t * 2 * np.pi)) / (2 * np.log(base))

    first, last = max(np.floor(index(high)), 0.0), np.ceil(index(low))
    keep = 1.0 - np.clip((i - first) / max(last - first, 0.001), 0.0, 1.0)
    return keep * f + (1 - keep) * f / factor, 1.0 + 0.1 * float(np.log(factor))


def rope_table(inv_freq, positions: int, mscale: float = 1.0, device="cuda", out=None):
    """Cosines and sines of every position below `positions` (float32
    [positions, rot / 2, 2], angles in float64, times mscale), made once."""
    f = np.ascontiguousarray(np.asarray(inv_freq, dtype=np.float64))
    if f.ndim != 1 or not 1 <= f.size <= 256:
        raise MxqError("inv_freq must hold 1 to 256 frequencies")
    if positions < 1:
        raise MxqError("positions must be at least 1")
    if out is None:
        out = torch.empty((positions, f.size, 2), dtype=torch.float32, device=device)
    _dev_array(out, positions * f.size * 2, torch.float32, "table", out.device)
    _check(lib().mxq_rope_table(f.ctypes.data_as(ctypes.c_void_p), 2 * f.size, positions,
                                float(mscale), _ptr(out), _current(out.device, "table")),
           "mxq_rope_table")
    return out


def _rotary(table, dev, interleaved: bool):
    if not (isinstance(table, torch.Tensor) and table.is_cuda and table.dtype is torch.float32
            and table.dim() == 3 and table.is_contiguous()):
        raise MxqError("the rotary table must be a contiguous float32 device tensor "
                       "[positions, rot / 2, 2]")
    n, half, two = table.shape
    if two != 2:
        raise MxqError("the rotary table is %s, not [positions, rot / 2, 2]" % (tuple(table.shape),))
    if table.device != dev:
        raise MxqError("the rotary table is on %s, not %s" % (table.device, dev))
    return ctypes.byref(_Rotary(table.data_ptr(), n, 2 * half, 1 if interleaved else 0))


def rope(x, pos, table, interleaved: bool = False, out=None):
    """Rotary positions on bf16 rows x [T, H, D] (strided) at positions pos (int32
    [T]): the first rot values of every head turn, as halves (i, i + rot / 2) or
    interleaved pairs (2 i, 2 i + 1).  `out` may be x (in place), else a tensor
    that does not overlap it."""
    T, H, D = _heads(x, "x")
    dev = x.device
    stream = _current(dev, "x")
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    elif out is not x and _heads(out, "out", dev, H, D)[0] != T:
        raise MxqError("out is %s, not %s" % (tuple(out.shape), tuple(x.shape)))
    st, so = x.stride(), out.stride()
    status = lib().mxq_rope(_rotary(table, dev, interleaved), x.data_ptr(), T, H, D, st[0], st[1],
                            _index(pos, T, torch.int32, "pos", dev), out.data_ptr(), so[0], so[1],
                            stream)
    if status:
        _check(status, "mxq_rope")
    return out


def rope_qk(q, k, pos, table, q_gain, k_gain, eps: float, interleaved: bool = False, q_out=None,
            k_out=None):
    """Queries q [T, Hq, D] and keys k [T, Hk, D] (bf16, strided; either may be None)
    normalised per head (x / sqrt(mean x^2 + eps) times its gain, bf16 [D]) and
    rotated as rope does, rounded once: (q_out, k_out).  Each may be its source (in
    place), else a tensor that overlaps none."""
    some = q if q is not None else k
    if some is None:
        raise MxqError("rope_qk needs q or k")
    T, H, D = _heads(some, "k" if q is None else "q")
    dev = some.device
    stream = _current(dev, "q or k")
    q_gain, q_out, q_args = _norm_side(q, H, q_gain, q_out, "q", T, D, dev)
    k_gain, k_out, k_args = _norm_side(k, H if q is None else None, k_gain, k_out, "k", T, D, dev)
    status = lib().mxq_rope_qk(_rotary(table, dev, interleaved),
                               ctypes.byref(_QkNorm(q_gain, k_gain, eps)),
                               _index(pos, T, torch.int32, "pos", dev), T, D, *q_args, *k_args,
                               stream)
    if status:
        _check(status, "mxq_rope_qk")
    return q_out, k_out


def _norm_side(x, H, gain, out, what: str, T: int, D: int, dev):
    """The gain, the result and the arguments of rope_qk's queries or keys (of H heads
    of checked rows, or None)."""
    if x is None:
        if out is not None:
            raise MxqError("%s_out needs %s" % (what, what))
        return None, None, (None, 0, 0, 0, None, 0, 0)
    if H is None:
        Tx, H, _ = _heads(x, what, dev, None, D)
        if Tx != T:
            raise MxqError("q and k have %d and %d tokens" % (T, Tx))
    if out is None:
        out = torch.empty((T, H, D), dtype=torch.bfloat16, device=dev)
    elif out is not x and _heads(out, what + "_out", dev, H, D)[0] != T:
        raise MxqError("%s_out is %s, not %s" % (what, tuple(out.shape), tuple(x.shape)))
    ts, hs, _ = x.stride()
    ots, ohs, _ = out.stride()
    return _index(gain, D, torch.bfloat16, what + "_gain", dev), out, (
        x.data_ptr(), H, ts, hs, out.data_ptr(), ots, ohs)


class PagedCache:
    """A paged MXINT KV cache of one layer (include/mxq.h mxq_paged_kv): `pages`
    pages of `page_tokens` tokens (a power of two, 16 to 1024) of Hkv heads of
    128 values.  k and v are (mant, exp) pairs of uint8 device tensors of
    pages * page_bytes and pages * page_exp_bytes bytes: the caller's, or new
    ones, zeroed."""

    def __init__(self, fmt: Format, Hkv: int, pages: int, page_tokens: int, device="cuda",
                 k=None, v=None):
        # (its own copy of the widths, which fix the buffers' sizes)
        self.fmt = Format(fmt.K, np.array(fmt.widths), fmt.perm, ("rne", "rna")[fmt.round],
                          ("sym", "full")[fmt.clamp])
        self.fmt.widths.setflags(write=False)
        fmt, self.Hkv = self.fmt, int(Hkv)
        self.pages, self.page_tokens = int(pages), int(page_tokens)
        L = lib()
        if not 16 <= self.page_tokens <= 1024:
            _check(2, "PagedCache")
        self.page_bytes = _size(L.mxq_kv_page_bytes(fmt.ref, self.Hkv, self.page_tokens),
                                "mxq_kv_page_bytes")
        self.page_exp_bytes = _size(L.mxq_kv_page_exp_bytes(fmt.ref, self.Hkv, self.page_tokens),
                                    "mxq_kv_page_exp_bytes")
        if self.pages < 1 or self.pages * self.page_tokens > 2 ** 31 - 1:
            _check(2, "PagedCache")

        def buffers(t, what):
            nm, ne = self.pages * self.page_bytes, self.pages * self.page_exp_bytes
            if t is None:
                return (torch.zeros(nm, dtype=torch.uint8, device=device),
                        torch.zeros(ne, dtype=torch.uint8, device=device))
            mant, exp = t
            _dev_bytes(mant, nm, what + " mantissa buffer")
            return mant, _dev_bytes(exp, ne, what + " exponent buffer", mant.device)

        self.k, self.v = buffers(k, "K"), buffers(v, "V")
        self.device = self.k[0].device
        if self.v[0].device != self.device:
            raise MxqError("K and V must be on one device")
        self._c = _PagedKv(self.pages, self.Hkv, self.page_tokens, 0, *[
            t.data_ptr() for t in self.k + self.v])
        self._ref = ctypes.byref(self._c)


def kv_append(cache: PagedCache, k, v, slots, pos=None, rope=None, interleaved: bool = False,
              q=None, q_out=None, q_gain=None, k_gain=None, eps: float = 0.0):
    """New tokens into the cache: keys k (rotated at positions pos int32 [T] with
    the table `rope`, where it is given) and values v, bf16 [T, Hkv, 128]
    (strided), quantized into slots (int64 [T], distinct; one outside the cache
    is padding).  With q (bf16 [T, Hq, 128], strided) the queries are rotated by
    the same launch, and returned (contiguous; q_out may be q if that is
    contiguous).  With k_gain (bf16 [128]; q_gain for the queries, and a `rope`) both
    are normalised per head before they turn, as rope_qk does."""
    dev = cache.device
    stream = _current(dev, "the cache")
    T = _heads(k, "k", dev, cache.Hkv, 128)[0]
    if _heads(v, "v", dev, cache.Hkv, 128)[0] != T:
        raise MxqError("k and v have %d and %d tokens" % (T, v.shape[0]))
    r = at = None
    if rope is not None:
        r = _rotary(rope, dev, interleaved)
        at = _index(pos, T, torch.int32, "pos", dev)
    Hq, qs, qp, op = 0, (0, 0), None, None
    if q is not None:
        Tq, Hq, _ = _heads(q, "q", dev, None, 128)
        if Tq != T or Hq < 1:
            raise MxqError("q is %s: %d tokens and a head are needed" % (tuple(q.shape), T))
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif _heads(q_out, "q_out", dev, Hq, 128)[0] != T or not q_out.is_contiguous():
            raise MxqError("q_out must be contiguous, [%d, %d, 128]" % (T, Hq))
        qs, qp, op = q.stride(), q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise MxqError("q_out needs q")
    ks, vs = k.stride(), v.stride()
    args = (k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], T,
            _index(slots, T, torch.int64, "slots", dev), at, r, qp, Hq, qs[0], qs[1], op, stream)
    if k_gain is None:
        if q_gain is not None:
            raise MxqError("q_gain needs k_gain")
        status = lib().mxq_kv_append(cache.fmt._ref, cache._ref, *args)
    else:
        if r is None or (q is None) != (q_gain is None):
            raise MxqError("gains need rope, and q_gain goes with q")
        norm = _QkNorm(None if q is None else _index(q_gain, 128, torch.bfloat16, "q_gain", dev),
                       _index(k_gain, 128, torch.bfloat16, "k_gain", dev), eps)
        status = lib().mxq_kv_append_norm(cache.fmt._ref, cache._ref, ctypes.byref(norm), *args)
    if status:
        _check(status, "mxq_kv_append")
    return q_out


def kv_read(cache: PagedCache, slots, out=None):
    """The cached rows of the slots (int64 [n]) as the bf16 values that they stand
    for: (k, v), each [n, Hkv, 128]; zeros for a slot outside the cache."""
    dev = cache.device
    stream = _current(dev, "the cache")
    n = slots.numel() if isinstance(slots, torch.Tensor) else 0
    at = _index(slots, n, torch.int64, "slots", dev)
    if out is None:
        # (one allocation for both)
        k, v = torch.empty((2, n, cache.Hkv, 128), dtype=torch.bfloat16, device=dev).unbind()
    else:
        k, v = out
        for t, what in ((k, "k"), (v, "v")):
            if _heads(t, what, dev, cache.Hkv, 128)[0] != n or not t.is_contiguous():
                raise MxqError("%s must be contiguous, [%d, %d, 128]" % (what, n, cache.Hkv))
    status = lib().mxq_kv_read(cache.fmt._ref, cache._ref, at, n, k.data_ptr(), v.data_ptr(), stream)
    if status:
        _check(status, "mxq_kv_read")
    return k, v


def attn_paged_work_bytes(cache: PagedCache, S: int, T: int, Hq: int, max_q: int,
                          max_kv: int) -> int:
    """Bytes of the scratch that attn_paged needs for these sizes."""
    return _size(lib().mxq_attn_paged_work_bytes(cache.fmt.ref, cache._ref, S, T, Hq, max_q,
                                                 max_kv), "mxq_attn_paged_work_bytes")


def attn_paged(q, cache: PagedCache, cu_q, kv_len, table, max_q: int, max_kv: int, scale: float,
               softcap: float = 0.0, window: int = 0, prefix=None, slopes=None, out=None,
               dtype=torch.bfloat16, work=None):
    """Attention of the new tokens of S sequences over their pages.  q: bf16 [T,
    Hq, 128] (strided), sequence s owning the rows cu_q[s] .. cu_q[s + 1] (int32
    [S + 1]), which are the last of its kv_len[s] (int32 [S]) cached tokens; its
    pages are table[s] (int32 [S, n]).  max_q and max_kv bound the sequences'
    rows and lengths (of more rows the first max_q are computed; the others, as
    rows of no sequence, stay as `out` holds them).  A row sees the tokens up to its own, of those the last
    `window` (0: all), and the first prefix[s] (int32 [S]); scores are capped by
    softcap * tanh(x / softcap) and lowered by slopes[h] (float32 [Hq]) times the
    distance.  Returns bf16 or float32 (`dtype`) [T, Hq, 128]: a bf16 result weighs
    the values with probabilities rounded to bf16 (and their sum, in float32), a
    float32 one with all their 24 bits, at up to twice the time."""
    dev = cache.device
    stream = _current(dev, "the cache")
    T, Hq, _ = _heads(q, "q", dev, None, 128)
    S = kv_len.numel() if isinstance(kv_len, torch.Tensor) else 0
    at = (_index(cu_q, S + 1, torch.int32, "cu_q", dev), _index(kv_len, S, torch.int32, "kv_len", dev))
    if not (isinstance(table, torch.Tensor) and table.is_cuda and table.dtype is torch.int32
            and table.dim() == 2 and table.shape[0] == S and table.device == dev
            and (table.stride(1) == 1 or table.shape[1] <= 1)):
        raise MxqError("table must be an int32 device tensor [%d, pages] with unit stride" % S)
    if prefix is not None:
        prefix = _index(prefix, S, torch.int32, "prefix", dev)
    if slopes is not None:
        slopes = _index(slopes, Hq, torch.float32, "slopes", dev)
    if out is None:
        if dtype is not torch.bfloat16 and dtype is not torch.float32:
            raise MxqError("dtype must be torch.bfloat16 or torch.float32")
        out = torch.empty_like(q, dtype=dtype, memory_format=torch.contiguous_format)
    elif not (isinstance(out, torch.Tensor) and out.is_cuda and out.is_contiguous()
              and out.dtype in (torch.bfloat16, torch.float32) and out.device == dev
              and out.shape == q.shape):
        raise MxqError("out must be a contiguous bf16 or float32 device tensor [%d, %d, 128]"
                       % (T, Hq))
    if work is None:
        n = attn_paged_work_bytes(cache, S, T, Hq, max_q, max_kv)
        work = torch.empty(max(n, 16), dtype=torch.uint8, device=dev)
    else:
        _dev_bytes(work, 0, "work", dev)
    batch = _PagedBatch(S, T, max_q, max_kv, at[0], at[1], table.data_ptr(), table.stride(0),
                        table.shape[1])
    opts = _AttnOpts(scale, softcap, window, prefix, slopes)
    qs = q.stride()
    status = lib().mxq_attn_paged(cache.fmt._ref, cache._ref, ctypes.byref(batch),
                                  ctypes.byref(opts), q.data_ptr(), Hq, qs[0], qs[1],
                                  out.data_ptr(), 1 if out.dtype is torch.float32 else 0,
                                  work.data_ptr(), work.numel(), stream)
    if status:
        _check(status, "mxq_attn_paged")
    return out


# --------------------------------------------------------------------------
# Layers with experts

def _bf16_or_f32(t, what: str, dim: int = 2):
    """A `dim`-D bf16 or float32 device tensor with unit column stride: whether float32."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == dim
            and t.dtype in (torch.bfloat16, torch.float32)
            and (t.stride(-1) == 1 or t.shape[-1] <= 1)):
        raise MxqError("%s must be a %d-D bf16 or float32 device tensor with unit column stride"
                       % (what, dim))
    return t.dtype is torch.float32


def _choices(t, dtype, what: str, dev, shape=None):
    """A contiguous 2-D device tensor [tokens, k]: its shape."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.dim() == 2
            and t.is_contiguous()):
        raise MxqError("%s must be a contiguous 2-D %s device tensor" % (what, dtype))
    if t.device != dev:
        raise MxqError("%s is on %s, not %s" % (what, t.device, dev))
    if shape is not None and t.shape != shape:
        raise MxqError("%s is %s, not %s" % (what, tuple(t.shape), tuple(shape)))
    return t.shape


def _bytes(t, n: int, what: str, dev):
    """The address of a contiguous uint8 tensor of at least n bytes on the device dev."""
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.uint8 and t.device == dev
            and t.is_contiguous() and t.numel() >= n):
        _dev_bytes(t, n, what, dev)
    return t.data_ptr()


def _image(out, fmt: Format, rows: int, dev):
    """The buffers of an image of `rows` rows (a multiple of 16), the caller's or new
    ones, and their addresses."""
    unit = fmt._units()
    if out is None:
        mant = torch.empty((rows >> 4) * unit[0], dtype=torch.uint8, device=dev)
        exp = torch.empty((rows >> 4) * unit[1], dtype=torch.uint8, device=dev)
        return (mant, exp), mant.data_ptr(), exp.data_ptr()
    mant, exp = out
    return out, _bytes(mant, (rows >> 4) * unit[0], "activation mantissa buffer", dev), _bytes(
        exp, (rows >> 4) * unit[1], "activation exponent buffer", dev)


class ExpertPlan:
    """Where the chosen token-expert pairs of a batch lie (include/mxq.h mxq_experts):
    `rows` rows of an operand image, expert e's from first[e] (int32 [experts + 1])
    on, row r holding pair[r] (int32 [rows], -1: none).  The buffers are new ones,
    with a scratch, which route or expert_plan fills; or the caller's, of a plan that
    is made (first and pair, and work, int32 [EXPERT_WORK * experts], where it is to be
    written again).  The sizes go by pairs and experts alone, so a plan serves every
    batch of as many tokens.  k: the pairs of a token; route and expert_plan set it with
    the plan that they write.  Where it is not known, the quantizers take any number of
    rows that divides the pairs for a row per token."""

    def __init__(self, pairs: int, experts: int, device="cuda", first=None, pair=None, work=None,
                 k=None):
        self.pairs, self.experts = int(pairs), int(experts)
        if k is not None and (k < 1 or self.pairs % k):
            raise MxqError("%d pairs are not %d for every token" % (self.pairs, k))
        self.k = k
        self.rows = _size(lib().mxq_expert_rows(self.pairs, self.experts), "mxq_expert_rows")
        if first is None and pair is None:
            # (one allocation; each part 16-byte aligned)
            at = self.experts + 4 & ~3
            n = EXPERT_WORK * self.experts
            whole = torch.empty(at + n + self.rows, dtype=torch.int32, device=device)
            first, work, pair = whole[:self.experts + 1], whole[at:at + n], whole[at + n:]
        elif first is None or pair is None:
            raise MxqError("a plan takes first and pair, or neither")
        self.device = first.device if isinstance(first, torch.Tensor) else None
        f = _index(first, self.experts + 1, torch.int32, "first", self.device)
        p = _index(pair, self.rows, torch.int32, "pair", self.device)
        w = None if work is None else _index(work, EXPERT_WORK * self.experts, torch.int32, "work",
                                             self.device)
        self.first, self.pair, self.work = first, pair, work
        self._c = _Experts(self.pairs, self.experts, 0, f, p, w)
        self._ref = ctypes.byref(self._c)


def route(logits, k: int, score: str = "softmax", normalise: bool = True, scale: float = 1.0,
          bias=None, out=None):
    """The k best of E experts for every token, from its scores logits (bf16 or
    float32 [T, E]), and their plan: (ids int32 [T, k], weights float32 [T, k],
    ExpertPlan).  score: "softmax" over all experts, or "sigmoid"; normalise:
    a token's weights are divided by their sum; bias (float32 [E]) is added to the
    score for the choice only; equal ones go to the lowest index.  out: such a
    triple, written."""
    f32 = _bf16_or_f32(logits, "logits")
    dev = logits.device
    stream = _current(dev, "logits")
    T, E = logits.shape
    if out is None:
        ids = torch.empty((T, k), dtype=torch.int32, device=dev)
        weights = torch.empty((T, k), dtype=torch.float32, device=dev)
        plan = ExpertPlan(T * k, E, device=dev, k=k)
    else:
        ids, weights, plan = out
        _choices(ids, torch.int32, "ids", dev, (T, k))
        _choices(weights, torch.float32, "weights", dev, (T, k))
        if plan.pairs != T * k or plan.experts != E or plan.device != dev:
            raise MxqError("the plan is of %d pairs and %d experts on %s, not %d and %d on %s"
                           % (plan.pairs, plan.experts, plan.device, T * k, E, dev))
    if bias is not None:
        bias = _index(bias, E, torch.float32, "bias", dev)
    if score not in _SCORES:
        raise MxqError("score must be 'softmax' or 'sigmoid'")
    opts = _RouteOpts(k, _SCORES[score], 1 if normalise else 0, scale, bias)
    status = lib().mxq_route(ctypes.byref(opts), logits.data_ptr(), 1 if f32 else 0, T,
                             logits.stride(0), ids.data_ptr(), weights.data_ptr(), plan._ref,
                             stream)
    if status:
        _check(status, "mxq_route")
    plan.k = k
    return ids, weights, plan


def expert_plan(ids, experts: int, out=None):
    """The plan of chosen experts ids (int32 [T, k], contiguous); ids outside [0,
    experts) are no choice.  out: an ExpertPlan, written."""
    T, k = _choices(ids, torch.int32, "ids", ids.device if isinstance(ids, torch.Tensor) else None)
    stream = _current(ids.device, "ids")
    if out is None:
        out = ExpertPlan(T * k, experts, device=ids.device)
    elif out.pairs != T * k or out.experts != experts or out.device != ids.device:
        raise MxqError("the plan is of %d pairs and %d experts on %s, not %d and %d on %s"
                       % (out.pairs, out.experts, out.device, T * k, experts, ids.device))
    _check(lib().mxq_expert_plan(ids.data_ptr(), out._ref, stream), "mxq_expert_plan")
    out.k = k or None
    return out


def _perms(perms, fmt: Format, experts: int, dev):
    if perms is None:
        return None
    if not (isinstance(perms, torch.Tensor) and perms.is_cuda and perms.dtype is torch.int32
            and perms.is_contiguous() and perms.shape == (experts, fmt.K)):
        raise MxqError("perms must be a contiguous int32 device tensor [%d, %d]" % (experts, fmt.K))
    if perms.device != dev:
        raise MxqError("perms is on %s, not %s" % (perms.device, dev))
    return perms.data_ptr()


def _per_row(rows: int, plan: ExpertPlan, what: str, dev) -> int:
    """Pairs per source row: as many as a token has, or one."""
    if plan.device != dev:
        raise MxqError("the plan is on %s, not %s" % (plan.device, dev))
    if rows == plan.pairs:
        return 1
    if rows == 0 or plan.pairs % rows or (plan.k is not None and rows * plan.k != plan.pairs):
        raise MxqError("%s has %d rows: a row per token (of %s pairs) or per pair (%d) is needed"
                       % (what, rows, plan.k or "some", plan.pairs))
    return plan.pairs // rows


def quantize_act_experts(x, fmt: Format, plan: ExpertPlan, perms=None, out=None):
    """quantize_act of bf16 rows x (a row per token, or per pair) by a plan: the
    operand image of its rows, for gemm_experts.  perms (int32 [experts, K]): a
    permutation for each expert in place of fmt's."""
    _bf16_2d(x, fmt.K, "activations")
    dev = x.device
    per = _per_row(x.shape[0], plan, "activations", dev)
    stream = _current(dev, "activations")
    out, mant, exp = _image(out, fmt, plan.rows, dev)
    status = lib().mxq_quantize_act_experts(fmt._ref, plan._ref, _perms(perms, fmt, plan.experts, dev),
                                            x.data_ptr(), per, x.stride(0), mant, exp, stream)
    if status:
        _check(status, "mxq_quantize_act_experts")
    return out


def quantize_act_swiglu_experts(gate, up, fmt: Format, plan: ExpertPlan, perms=None, out=None):
    """quantize_act_swiglu of gate and up (a row per pair, as gemm_experts gives
    them, or per token) by a plan."""
    _bf16_2d(gate, fmt.K, "gate")
    _bf16_2d(up, fmt.K, "up")
    if up.shape != gate.shape or up.stride() != gate.stride():
        raise MxqError("gate and up must have the same shape and strides")
    if up.device != gate.device:
        raise MxqError("gate and up must be on one device")
    dev = gate.device
    per = _per_row(gate.shape[0], plan, "gate", dev)
    stream = _current(dev, "gate")
    out, mant, exp = _image(out, fmt, plan.rows, dev)
    status = lib().mxq_quantize_act_swiglu_experts(
        fmt._ref, plan._ref, _perms(perms, fmt, plan.experts, dev), gate.data_ptr(), up.data_ptr(),
        per, gate.stride(0), mant, exp, stream)
    if status:
        _check(status, "mxq_quantize_act_swiglu_experts")
    return out


def pack_experts(w, fmt: Format, perms=None):
    """pack_weights of every expert's weights w (bf16 [experts, N, >= K]), one after
    the other: (mant uint8 [experts, weight_bytes(N)], exp uint8 [experts,
    weight_exp_bytes(N)])."""
    if not (isinstance(w, torch.Tensor) and w.is_cuda and w.dim() == 3):
        raise MxqError("weights must be a 3-D bf16 device tensor [experts, N, K]")
    E, N, _ = w.shape
    stream = _current(w.device, "weights")
    _perms(perms, fmt, E, w.device)
    mant = torch.empty((E, fmt.weight_bytes(N)), dtype=torch.uint8, device=w.device)
    exp = torch.empty((E, fmt.weight_exp_bytes(N)), dtype=torch.uint8, device=w.device)
    for e in range(E):
        f = fmt if perms is None else Format(fmt.K, fmt.widths, perms[e], ("rne", "rna")[fmt.round],
                                             ("sym", "full")[fmt.clamp])
        _check(lib().mxq_pack_weights(f.ref, _ptr(_bf16_2d(w[e], fmt.K, "weights")), N, w.stride(1),
                                      _ptr(mant[e]), _ptr(exp[e]), stream), "mxq_pack_weights")
    return mant, exp


def gemm_experts(a_mant, a_exp, w_mant, w_exp, fmt: Format, plan: ExpertPlan, N: int, out=None,
                 dtype=torch.bfloat16):
    """Every pair's row times its expert's weights (pack_experts): [pairs, N], bf16
    or float32 (`dtype`); rows of pairs that chose no expert stay as `out` holds
    them.  bf16 rows are what quantize_act_swiglu_experts takes; for rows that
    combine_experts adds up float32 spares each a rounding before the sum."""
    dev = plan.device
    stream = _current(dev, "the plan")
    if N < 0:
        raise MxqError("N must be non-negative")
    unit, tiles, slabs = fmt._units(), plan.rows >> 4, plan.experts * (N + 127 >> 7)
    at = (_bytes(a_mant, tiles * unit[0], "a_mant", dev), _bytes(a_exp, tiles * unit[1], "a_exp", dev),
          _bytes(w_mant, slabs * unit[2], "w_mant", dev), _bytes(w_exp, slabs * unit[3], "w_exp", dev))
    if out is None:
        if dtype is not torch.bfloat16 and dtype is not torch.float32:
            raise MxqError("dtype must be torch.bfloat16 or torch.float32")
        out = torch.empty((plan.pairs, N), dtype=dtype, device=dev)
        f32 = dtype is torch.float32
    else:
        f32 = _bf16_or_f32(out, "out")
        if out.device != dev or out.shape[0] < plan.pairs or out.shape[1] < N:
            raise MxqError("out is %s on %s, smaller than [%d, %d] or not on %s"
                           % (tuple(out.shape), out.device, plan.pairs, N, dev))
    status = lib().mxq_gemm_experts(fmt._ref, plan._ref, N, *at, out.data_ptr(), 1 if f32 else 0,
                                    out.stride(0), stream)
    if status:
        _check(status, "mxq_gemm_experts")
    return out


def combine_experts(y, ids, weights, plan: ExpertPlan, residual=None, out=None,
                    dtype=torch.bfloat16):
    """A token's weighted sum over its experts' rows of y (bf16 or float32 [T * k,
    N]), on top of residual (bf16 [T, N]) where it is given: bf16 or float32
    (`dtype`) [T, N].  out may be residual."""
    f32 = _bf16_or_f32(y, "y")
    dev = y.device
    stream = _current(dev, "y")
    T, k = shape = _choices(ids, torch.int32, "ids", dev)
    _choices(weights, torch.float32, "weights", dev, shape)
    rows, N = y.shape
    if T * k != plan.pairs or rows < plan.pairs:
        raise MxqError("y has %d rows and ids %d pairs, the plan %d" % (rows, T * k, plan.pairs))
    if plan.k is not None and k != plan.k:
        raise MxqError("ids have %d pairs a token, the plan %d" % (k, plan.k))
    r = ldr = 0
    if residual is not None:
        if _bf16_or_f32(residual, "residual") or residual.device != dev:
            raise MxqError("residual must be bf16, on %s" % dev)
        if residual.shape != (T, N):
            raise MxqError("residual is %s, not [%d, %d]" % (tuple(residual.shape), T, N))
        r, ldr = residual.data_ptr(), residual.stride(0)
    if out is None:
        if dtype is not torch.bfloat16 and dtype is not torch.float32:
            raise MxqError("dtype must be torch.bfloat16 or torch.float32")
        out = torch.empty((T, N), dtype=dtype, device=dev)
        of32 = dtype is torch.float32
    else:
        of32 = _bf16_or_f32(out, "out")
        if out.device != dev or out.shape != (T, N):
            raise MxqError("out is %s on %s, not [%d, %d] on %s"
                           % (tuple(out.shape), out.device, T, N, dev))
    status = lib().mxq_combine_experts(y.data_ptr(), 1 if f32 else 0, y.stride(0), ids.data_ptr(),
                                       weights.data_ptr(), T, k, plan.experts, N, r, ldr,
                                       out.data_ptr(), 1 if of32 else 0, out.stride(0), stream)
    if status:
        _check(status, "mxq_combine_experts")
    return out

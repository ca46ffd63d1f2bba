"""Thin ctypes binding of libpuro (include/puro.h): argument marshalling only.

Every operation runs in the HIP kernels of ``libpuro.so``; torch supplies
device memory and the current stream. There is no fallback: if the library
is missing or a call fails, an exception is raised.

Tensors: BF16 data as ``torch.bfloat16`` (or int16/uint16 holding the bit
patterns), FP8 codes as ``torch.uint8``, scales as ``torch.float32``, all on
the GPU; 2-D with unit stride along rows.
"""

import ctypes
import functools
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpuro.so")

E4M3, E5M2 = 0, 1
SCALE_TENSOR, SCALE_ROW_1x128, SCALE_COL_128x1, SCALE_BLOCK_128x128 = 0, 1, 2, 3
SCALE_KMAJOR = 0x100    # OR-ed into a grouped mode: k-block-major scale arrays
SCALE_FP32, SCALE_POW2, SCALE_POW2_FLOOR = 0, 1, 2
OUT_BF16, OUT_FP32 = 0, 1

_i64, _sz, _p, _i = ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int


class PuroError(RuntimeError):
    def __init__(self, fn, code, msg):
        super().__init__("%s failed: %s (status %d)" % (fn, msg, code))
        self.code = code


class Operand(ctypes.Structure):
    """puro_fp8_operand: FP8 codes [rows, K] (row pitch ld bytes) and scales."""
    _fields_ = [("data", _p), ("ld", _i64), ("fmt", _i), ("mode", _i), ("scale", _p)]


class Heads(ctypes.Structure):
    """puro_heads: where the heads of a [batch, seq, heads, head_dim] tensor are."""
    _fields_ = [("data", _p), ("batch_stride", _i64), ("row_stride", _i64), ("head_stride", _i64)]


class RopeArgs(ctypes.Structure):
    """puro_rope."""
    _fields_ = [("table", _p), ("len", _i64), ("dim", _i), ("interleaved", _i), ("positions", _p)]


class Recipe(ctypes.Structure):
    """puro_linear_recipe."""
    _fields_ = [("x_fmt", _i), ("w_fmt", _i), ("dy_fmt", _i), ("blockwise", _i), ("rnd", _i)]


class Saved(ctypes.Structure):
    """puro_linear_saved."""
    _fields_ = [("xq_t", _p), ("x_scale", _p), ("wq_t", _p), ("w_scale", _p)]


_HEADS, _ROPE = ctypes.POINTER(Heads), ctypes.POINTER(RopeArgs)

_SIGS = {
    "puro_status_string": (ctypes.c_char_p, [_i]),
    "puro_amax_workspace_size": (_sz, [_i64, _i64]),
    "puro_amax": (_i, [_p, _i64, _i64, _i64, _p, _p, _sz, _p]),
    "puro_quantize_workspace_size": (_sz, [_i64, _i64]),
    "puro_quantize_fp8": (_i, [_p, _i64, _i64, _i64, _i, _i, _i, _p, _p, _p, _p, _p, _p, _sz, _p]),
    "puro_quantize_fp8_static": (_i, [_p, _i64, _i64, _i64, _i, _i, _i, _p, _p, _p, _p, _p, _p]),
    "puro_swiglu_quantize_workspace_size": (_sz, [_i64, _i64]),
    "puro_swiglu_quantize_fp8": (_i, [_p, _i64, _i64, _i64, _i, _i, _i, _p, _p, _p, _p, _p, _sz, _p]),
    "puro_swiglu_bwd_quantize_workspace_size": (_sz, [_i64, _i64]),
    "puro_swiglu_bwd_quantize_fp8": (_i, [_p, _i64, _p, _i64, _i64, _i64, _i, _i, _i, _p, _p, _p, _p, _p, _sz, _p]),
    "puro_rmsnorm_quantize_workspace_size": (_sz, [_i64, _i64]),
    "puro_rmsnorm_quantize_fp8": (_i, [_p, _p, _i64, _i64, _i64, ctypes.c_float, _i, _i, _i, _p, _p, _p, _p, _p,
                                       _p, _sz, _p]),
    "puro_rope_table": (_i, [_p, _i64, _i, ctypes.c_double, _p]),
    "puro_qk_norm_rope_fwd": (_i, [_i64, _i64, _i, _i, _i, _HEADS, _HEADS, _p, _p, ctypes.c_float, _ROPE, _HEADS,
                                   _HEADS, _p]),
    "puro_qk_norm_rope_bwd_workspace_size": (_sz, [_i64, _i64, _i]),
    "puro_qk_norm_rope_bwd": (_i, [_i64, _i64, _i, _i, _i] + [_HEADS] * 5 + [_p, _p, ctypes.c_float, _ROPE]
                              + [_HEADS] * 3 + [_p, _p, _p, _sz, _p]),
    "puro_qk_norm_rope_bwd_quantize_workspace_size": (_sz, [_i64, _i64, _i, _i, _i]),
    "puro_qk_norm_rope_bwd_quantize_fp8": (_i, [_i64, _i64, _i, _i, _i] + [_HEADS] * 5 + [_p, _p, ctypes.c_float, _ROPE]
                                           + [_i, _i, _i, _p, _p, _p, _p, _p, _p, _p, _sz, _p]),
    "puro_fp8_gemm_workspace_size": (_sz, [_i64, _i64, _i64, _i]),
    "puro_fp8_gemm_plan": (_i, [_i64, _i64, _i64, _i, _i, ctypes.POINTER(_i), ctypes.POINTER(_i),
                                ctypes.POINTER(_i), ctypes.POINTER(_i), ctypes.POINTER(_i)]),
    "puro_fp8_gemm": (_i, [_i64, _i64, _i64, ctypes.POINTER(Operand), ctypes.POINTER(Operand),
                           _p, _i, _i64, _i, _p, _sz, _p]),
    "puro_fp8_gemm_epilogue": (_i, [_i64, _i64, _i64, ctypes.POINTER(Operand), ctypes.POINTER(Operand),
                                    _p, _i64, _p, _p, _i64, _p, _sz, _p]),
    "puro_linear_saved_bytes": (_sz, [_i64, _i64, _i64, ctypes.POINTER(Recipe), ctypes.POINTER(_sz * 4)]),
    "puro_linear_fwd_workspace_size": (_sz, [_i64, _i64, _i64, ctypes.POINTER(Recipe)]),
    "puro_linear_bwd_workspace_size": (_sz, [_i64, _i64, _i64, ctypes.POINTER(Recipe)]),
    "puro_linear_fwd": (_i, [_p, _p, _i64, _i64, _i64, ctypes.POINTER(Recipe), _p, ctypes.POINTER(Saved),
                             _p, _sz, _p]),
    "puro_linear_bwd": (_i, [_p, ctypes.POINTER(Saved), _i64, _i64, _i64, ctypes.POINTER(Recipe), _p, _p,
                             _i, _p, _sz, _p]),
    "puro_lm_head_ce_workspace_size": (_sz, [_i64, _i64, _i64, _i, _i]),
    "puro_lm_head_ce_fwd": (_i, [_p, _p, _p, _i64, _i64, _i64, _i, _p, _p, _p, _sz, _p]),
    "puro_lm_head_ce_bwd": (_i, [_p, _p, _p, _p, _i64, _i64, _i64, _i, ctypes.c_float, _p, _p, _p, _sz, _p]),
    "puro_lm_head_distill_workspace_size": (_sz, [_i64, _i64, _i64, _i64, _i]),
    "puro_lm_head_distill_fwd": (_i, [_p, _p, _p, _p, _i64, _i64, _i64, _i64, _i, ctypes.c_float, _p, _p, _p, _p, _sz, _p]),
    "puro_lm_head_distill_bwd": (_i, [_p, _p, _p, _p, _p, _p, _i64, _i64, _i64, _i64, _i, ctypes.c_float, _p,
                                      ctypes.c_float, _p, _p, _i, _i, _p, _sz, _p]),
    "puro_quantize_int8_workspace_size": (_sz, [_i64, _i64]),
    "puro_quantize_int8": (_i, [_p, _i64, _i64, _i64, _p, _p, _p, _i64, _p, _p, _sz, _p]),
    "puro_rmsnorm_quantize_int8": (_i, [_p, _p, _i64, _i64, _i64, ctypes.c_float, _p, _p, _p, _p]),
    "puro_swiglu_quantize_int8": (_i, [_p, _i64, _i64, _i64, _p, _p, _p]),
    "puro_int8_gemm_workspace_size": (_sz, [_i64, _i64, _i64]),
    "puro_int8_gemm": (_i, [_i64, _i64, _i64, _p, _i64, _p, _p, _i64, _p, _p, _i, _i64, _i, _p, _p, _i64, _p, _sz, _p]),
    "puro_int8_linear_fwd_workspace_size": (_sz, [_i64, _i64, _i64]),
    "puro_int8_linear_bwd_workspace_size": (_sz, [_i64, _i64, _i64]),
    "puro_int8_linear_fwd": (_i, [_p, _p, _i64, _i64, _i64, _p, ctypes.POINTER(Saved), _p, _sz, _p]),
    "puro_int8_linear_bwd": (_i, [_p, ctypes.POINTER(Saved), _i64, _i64, _i64, _p, _p, _i, _p, _sz, _p]),
    "puro_verify_drafts_workspace_size": (_sz, [_i64, _i64, _i64, _i64]),
    "puro_verify_drafts": (_i, [_i64, _i64, _i64, _i64, _i, _i, _p, _i64, _p, _i64, _p, _p, _p, _p, ctypes.c_double, _p, _p,
                                _p, _sz, _p]),
    "puro_muonh_workspace_size": (_sz, [_i64, _i64, _i64]),
    "puro_muonh_step": (_i, [_i64, _i64, _i64, _p, _p, _p, _p, _p, ctypes.c_float, _i, ctypes.c_float, _i, _p,
                             _p, _sz, _p]),
    "puro_newton_schulz_workspace_size": (_sz, [_i64, _i64, _i64]),
    "puro_newton_schulz_bf16": (_i, [_i64, _i64, _i64, _p, _i, _p, _p, _sz, _p]),
}

_lib = None


def lib():
    """The loaded libpuro (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libpuro.so is not built (run paper_2608_27370_amd/build.py or "
                              "__graft_entry__.build()); there is no fallback path")
        l = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(l, name)
            f.restype = res
            f.argtypes = args
        _lib = l
    return _lib


def status_string(code):
    return lib().puro_status_string(code).decode()


def _check(fn, code):
    if code != 0:
        raise PuroError(fn, code, status_string(code))


def _ptr(t):
    return None if t is None else t.data_ptr()


# torch's raw handle of the current stream of a device, without the Stream
# object that torch.cuda.current_stream() builds around it (2 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


# Workspace sizes depend on the sizes alone; a program calls with few of them.
# (typed: 1, 1.0 and True are different arguments to ctypes, which refuses 1.0)
@functools.lru_cache(maxsize=1024, typed=True)
def _size(fn, *args):
    return getattr(lib(), fn)(*args)


def _ld(t):
    assert t.dim() == 2, "2-D tensors"
    if t.numel() == 0:
        return t.shape[1]          # torch gives empty tensors zero strides
    assert t.stride(1) == 1, "2-D tensors with unit column stride"
    return t.stride(0)


def _ws(nbytes, ws, device):
    if nbytes == 0:
        return None, 0
    if ws is None:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    assert ws.numel() * ws.element_size() >= nbytes
    return ws, ws.numel() * ws.element_size()


# ------------------------------------------------------------------- amax
def amax(x, out=None, ws=None):
    """max |x| of a 2-D BF16 tensor as a one-element float32 device tensor."""
    rows, cols = x.shape
    if out is None:
        out = torch.empty(1, dtype=torch.float32, device=x.device)
    w, nb = _ws(lib().puro_amax_workspace_size(rows, cols), ws, x.device)
    _check("puro_amax", lib().puro_amax(_ptr(x), rows, cols, _ld(x), _ptr(out), _ptr(w), nb, _stream()))
    return out


# --------------------------------------------------------------- quantise
def quantize_fp8(x, fmt, mode=SCALE_TENSOR, rnd=SCALE_FP32, amax_in=None, want_q=True, want_qT=False,
                 out=None, ws=None):
    """Quantise a 2-D BF16 tensor; returns dict(q, scale, qT, scaleT) (absent
    outputs are None). ``out`` may supply preallocated outputs."""
    rows, cols = x.shape
    dev = x.device
    q, scale, qT, scaleT = _quant_outputs(rows, cols, mode, want_q, want_qT, out, dev)
    w, nb = _ws(_size("puro_quantize_workspace_size", rows, cols), ws, dev)
    _check("puro_quantize_fp8", lib().puro_quantize_fp8(
        _ptr(x), rows, cols, _ld(x), fmt, mode, rnd, _ptr(amax_in), _ptr(q), _ptr(scale), _ptr(qT),
        _ptr(scaleT), _ptr(w), nb, _stream()))
    return dict(q=q, scale=scale, qT=qT, scaleT=scaleT)


def quantize_fp8_static(x, fmt, mode=SCALE_TENSOR, rnd=SCALE_FP32, amax_in=None, want_q=True, want_qT=False,
                        out=None):
    """quantize_fp8 through the allocation-free entry point (the library's
    own per-GPU scratch instead of a workspace); pass preallocated ``out``
    tensors to allocate nothing at all."""
    rows, cols = x.shape
    q, scale, qT, scaleT = _quant_outputs(rows, cols, mode, want_q, want_qT, out, x.device)
    _check("puro_quantize_fp8_static", lib().puro_quantize_fp8_static(
        _ptr(x), rows, cols, _ld(x), fmt, mode, rnd, _ptr(amax_in), _ptr(q), _ptr(scale), _ptr(qT),
        _ptr(scaleT), _stream()))
    return dict(q=q, scale=scale, qT=qT, scaleT=scaleT)


def _quant_outputs(rows, cols, mode, want_q, want_qT, out, dev):
    """Output tensors of a quantisation (supplied ones from `out` kept), in the
    scale layout the mode's SCALE_KMAJOR flag selects."""
    out = dict(out) if out else {}
    G = 128
    km = bool(mode & SCALE_KMAJOR)
    base = mode & ~SCALE_KMAJOR
    if base == SCALE_COL_128x1:
        want_q, want_qT = False, True
    q = out.get("q") if want_q else None
    if want_q and q is None:
        q = torch.empty(rows, cols, dtype=torch.uint8, device=dev)
    qT = out.get("qT") if want_qT else None
    if want_qT and qT is None:
        qT = torch.empty(cols, rows, dtype=torch.uint8, device=dev)
    scale, scaleT = out.get("scale"), out.get("scaleT")

    def new(shape):
        return torch.empty(*(shape[::-1] if km else shape), dtype=torch.float32, device=dev)
    if base == SCALE_TENSOR:
        scale = scale if scale is not None else torch.empty(1, dtype=torch.float32, device=dev)
        scaleT = None
    elif base == SCALE_ROW_1x128:
        scale = scale if scale is not None else new((rows, cols // G))
        if want_qT and scaleT is None:
            scaleT = new((cols, rows // G))
    elif base == SCALE_COL_128x1:
        scale = None
        scaleT = scaleT if scaleT is not None else new((cols, rows // G))
    elif base == SCALE_BLOCK_128x128:
        scale = scale if scale is not None else new((rows // G, cols // G))
        if want_qT and scaleT is None:
            scaleT = new((cols // G, rows // G))
    if not want_qT:
        scaleT = None
    return q, scale, qT, scaleT


# -------------------------------------------- SwiGLU backward + quantise
def swiglu_bwd_quantize_fp8(dh, gu, fmt, mode=SCALE_TENSOR, rnd=SCALE_FP32, want_q=True, want_qT=False,
                            out=None, ws=None):
    """Quantise dgu = [dH u silu'(g) | dH silu(g)] [rows, 2 cols] from dH
    [rows, cols] and the saved gate/up output gu [rows, 2 cols] without
    writing dgu; returns dict(q, scale, qT, scaleT)."""
    rows, cols = dh.shape
    assert gu.shape[0] == rows and gu.shape[1] >= 2 * cols
    dev = dh.device
    q, scale, qT, scaleT = _quant_outputs(rows, 2 * cols, mode, want_q, want_qT, out, dev)
    w, nb = _ws(_size("puro_swiglu_bwd_quantize_workspace_size", rows, cols), ws, dev)
    _check("puro_swiglu_bwd_quantize_fp8", lib().puro_swiglu_bwd_quantize_fp8(
        _ptr(dh), _ld(dh), _ptr(gu), _ld(gu), rows, cols, fmt, mode, rnd, _ptr(q), _ptr(scale), _ptr(qT),
        _ptr(scaleT), _ptr(w), nb, _stream()))
    return dict(q=q, scale=scale, qT=qT, scaleT=scaleT)


# ---------------------------------------------------- RMSNorm + quantise
def rmsnorm_quantize_fp8(x, gamma, eps, fmt, mode=SCALE_TENSOR, rnd=SCALE_FP32, want_q=True, want_qT=False,
                         out=None, ws=None):
    """Quantise y = BF16(x * rstd * gamma) (RMSNorm of each row of x) without
    writing y; returns dict(q, scale, qT, scaleT, rstd) with rstd [rows]
    float32 (out may also supply "rstd")."""
    rows, cols = x.shape
    dev = x.device
    q, scale, qT, scaleT = _quant_outputs(rows, cols, mode, want_q, want_qT, out, dev)
    rstd = (out or {}).get("rstd")
    if rstd is None:
        rstd = torch.empty(rows, dtype=torch.float32, device=dev)
    w, nb = _ws(_size("puro_rmsnorm_quantize_workspace_size", rows, cols), ws, dev)
    _check("puro_rmsnorm_quantize_fp8", lib().puro_rmsnorm_quantize_fp8(
        _ptr(x), _ptr(gamma), rows, cols, _ld(x), float(eps), fmt, mode, rnd, _ptr(q), _ptr(scale), _ptr(qT),
        _ptr(scaleT), _ptr(rstd), _ptr(w), nb, _stream()))
    return dict(q=q, scale=scale, qT=qT, scaleT=scaleT, rstd=rstd)


# ----------------------------------------------------- SwiGLU + quantise
def swiglu_quantize_fp8(gu, cols, fmt, mode=SCALE_TENSOR, rnd=SCALE_FP32, want_q=True, want_qT=False,
                        out=None, ws=None):
    """Quantise H = BF16(silu(gate) * up) of a fused gate/up output gu
    [rows, 2 cols] (gate = gu[:, :cols], up = gu[:, cols:2 cols]) without
    writing H; returns dict(q, scale, qT, scaleT) as quantize_fp8 does."""
    rows = gu.shape[0]
    assert gu.shape[1] >= 2 * cols
    dev = gu.device
    q, scale, qT, scaleT = _quant_outputs(rows, cols, mode, want_q, want_qT, out, dev)
    w, nb = _ws(_size("puro_swiglu_quantize_workspace_size", rows, cols), ws, dev)
    _check("puro_swiglu_quantize_fp8", lib().puro_swiglu_quantize_fp8(
        _ptr(gu), rows, cols, _ld(gu), fmt, mode, rnd, _ptr(q), _ptr(scale), _ptr(qT), _ptr(scaleT),
        _ptr(w), nb, _stream()))
    return dict(q=q, scale=scale, qT=qT, scaleT=scaleT)


# ------------------------------- query / key norm with position rotation
# (these calls take few microseconds on the GPU, so their checks are few operations each)
def _check_tensor(t, what, dtypes, device):
    """A tensor whose memory a kernel may take: its type, and its device the current one (whose stream runs it)."""
    if t.dtype not in dtypes:
        raise TypeError("%s: %s expected, got %s" % (what, " or ".join(str(d) for d in dtypes), t.dtype))
    if t.get_device() != device:
        raise ValueError("%s is on %s, the current device is cuda:%d" % (what, t.device, device))


_BF16_BITS = (torch.bfloat16, torch.int16, torch.uint16)
_FP32, _INT32 = (torch.float32,), (torch.int32,)
_current = torch.cuda.current_device


@dataclass
class Rope:
    """The position rotation: table [length, dim / 2, 2] FP32 of (cos, sin) per position and pair (``rope_table``
    makes one; a scaled or interpolated one does as well), pairs (i, i + dim / 2) or, interleaved, (2 i, 2 i + 1)."""
    table: torch.Tensor
    interleaved: bool = False

    @property
    def dim(self):
        return 2 * self.table.shape[1]


def rope_table(length, dim, theta=1e6, interleaved=False, device=None):
    """The rotation by angles p theta^(-2 i / dim) at positions p < length (angles in double precision)."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    table = torch.empty(length, dim // 2, 2, dtype=torch.float32, device=device)
    _check_tensor(table, "table", _FP32, _current())
    _check("puro_rope_table", lib().puro_rope_table(_ptr(table), length, dim, float(theta), _stream()))
    return Rope(table, interleaved)


def _rope_args(rope, positions, tokens, device):
    if rope is None:
        return None
    t = rope.table
    n, half, two = t.shape
    if two != 2 or not t.is_contiguous():
        raise ValueError("the rotation's table is a contiguous [length, dim / 2, 2] tensor")
    if t.dtype != torch.float32 or t.get_device() != device:
        _check_tensor(t, "table", _FP32, device)
    if positions is not None:
        if positions.dtype != torch.int32 or positions.get_device() != device:
            _check_tensor(positions, "positions", _INT32, device)
        if positions.numel() != tokens or not positions.is_contiguous():
            raise ValueError("positions: one for each of the %d tokens, contiguous" % tokens)
        positions = positions.data_ptr()
    return RopeArgs(t.data_ptr(), n, 2 * half, 1 if rope.interleaved else 0, positions)


def _heads(t, what, shape, device):
    """Heads [S, H, D] or [B, S, H, D] of any strides (D contiguous)."""
    if t.shape != shape:
        raise ValueError("%s: shape %s expected, got %s" % (what, tuple(shape), tuple(t.shape)))
    if t.dtype not in _BF16_BITS or t.get_device() != device:
        _check_tensor(t, what, _BF16_BITS, device)
    *batch, row, head, one = t.stride()
    if one != 1 and t.numel() > 0 and shape[-1] > 1:
        raise ValueError("%s: the values of a head are contiguous" % what)
    return Heads(t.data_ptr(), batch[0] if batch else 0, row, head)


def _new_heads(like, seq, heads, d):
    """A new contiguous tensor of the shape of `like`, and its Heads."""
    t = torch.empty_like(like, memory_format=torch.contiguous_format)
    return t, Heads(t.data_ptr(), seq * heads * d, heads * d, d)


def _qk_sizes(q, k):
    """(batch, seq, heads_q, heads_k, head_dim) of q [.., S, Hq, D] and k [.., S, Hk, D]."""
    a, b = q.shape, k.shape
    if len(a) == 3 and len(b) == 3:
        a, b = (1, *a), (1, *b)
    if len(a) != 4 or len(b) != 4:
        raise ValueError("heads are [S, H, D] or [B, S, H, D], both kinds alike")
    batch, seq, hq, d = a
    batch_k, seq_k, hk, d_k = b
    if batch != batch_k or seq != seq_k or d != d_k:
        raise ValueError("q %s and k %s differ in more than their heads" % (tuple(q.shape), tuple(k.shape)))
    return batch, seq, hq, hk, d


def _gamma(g, what, d, device):
    if g is None:
        return None
    if g.dtype not in _BF16_BITS or g.get_device() != device:
        _check_tensor(g, what, _BF16_BITS, device)
    if g.numel() != d or not g.is_contiguous():
        raise ValueError("%s: %d contiguous values" % (what, d))
    return g.data_ptr()


def qk_norm_rope_fwd(q, k, gamma_q=None, gamma_k=None, rope=None, positions=None, eps=1e-6, q_out=None, k_out=None):
    """RMSNorm (weights gamma [D], None: no norm) of every query and key head and the rotation by its token's
    position (None: no rotation; positions None: a token's place in its sequence). q [.., S, Hq, D], k [.., S, Hk, D]
    BF16 of any strides, for instance views of the QKV projection's output; returns (q_out, k_out), new contiguous
    tensors or those given (which may be q and k themselves)."""
    batch, seq, hq, hk, d = _qk_sizes(q, k)
    dev = _current()
    a, b = _heads(q, "q", q.shape, dev), _heads(k, "k", k.shape, dev)
    q_out, aq = _new_heads(q, seq, hq, d) if q_out is None else (q_out, _heads(q_out, "q_out", q.shape, dev))
    k_out, ak = _new_heads(k, seq, hk, d) if k_out is None else (k_out, _heads(k_out, "k_out", k.shape, dev))
    _check("puro_qk_norm_rope_fwd", lib().puro_qk_norm_rope_fwd(
        batch, seq, hq, hk, d, a, b, _gamma(gamma_q, "gamma_q", d, dev), _gamma(gamma_k, "gamma_k", d, dev), eps,
        _rope_args(rope, positions, batch * seq, dev), aq, ak, _stream()))
    return q_out, k_out


def _dgamma(gamma, want, d, device):
    return torch.empty(d, dtype=torch.float32, device=device) if want and gamma is not None else None


def _qk_grads(dq, dk, dv, q, k, gamma_q, gamma_k, rope, positions, eps, sizes, dev):
    """The leading arguments of both backward calls."""
    d, sq, sk = sizes[4], dq.shape, dk.shape
    return (*sizes, _heads(dq, "dq", sq, dev), _heads(dk, "dk", sk, dev),
            _heads(dv, "dv", sk, dev) if dv is not None else None, _heads(q, "q", sq, dev), _heads(k, "k", sk, dev), _gamma(gamma_q, "gamma_q", d, dev), _gamma(gamma_k, "gamma_k", d, dev), eps,
            _rope_args(rope, positions, sizes[0] * sizes[1], dev))


def qk_norm_rope_bwd(dq, dk, dv, q, k, gamma_q=None, gamma_k=None, rope=None, positions=None, eps=1e-6, out=None,
                     want_dgamma=True, ws=None):
    """The gradient dqkv [tokens, (Hq + 2 Hk) D] (BF16) of the QKV projection's output, from the gradients of the
    rotated heads and of the value heads ([.., S, H, D], any strides; dv None: [tokens, (Hq + Hk) D] without them),
    and dgamma_q, dgamma_k [D] (FP32; None where there is no weight). q and k are the forward's inputs."""
    batch, seq, hq, hk, d = sizes = _qk_sizes(dq, dk)
    dev = _current()
    args = _qk_grads(dq, dk, dv, q, k, gamma_q, gamma_k, rope, positions, eps, sizes, dev)
    tokens, width = batch * seq, (hq + (2 if dv is not None else 1) * hk) * d
    if out is None:
        out, ld = dq.new_empty(tokens, width), width
    else:
        if out.shape != (tokens, width):
            raise ValueError("out: shape %s expected, got %s" % ((tokens, width), tuple(out.shape)))
        _check_tensor(out, "out", _BF16_BITS, dev)
        ld = _ld(out)
    at = out.data_ptr()
    dgq, dgk = _dgamma(gamma_q, want_dgamma, d, dq.device), _dgamma(gamma_k, want_dgamma, d, dq.device)
    nb = 0
    if dgq is not None or dgk is not None:
        ws, nb = _ws(_size("puro_qk_norm_rope_bwd_workspace_size", batch, seq, d), ws, dq.device)
    _check("puro_qk_norm_rope_bwd", lib().puro_qk_norm_rope_bwd(
        *args, Heads(at, ld * seq, ld, d), Heads(at + 2 * hq * d, ld * seq, ld, d),
        Heads(at + 2 * (hq + hk) * d, ld * seq, ld, d) if dv is not None else None, _ptr(dgq), _ptr(dgk),
        _ptr(ws) if nb else None, nb, _stream()))
    return out, dgq, dgk


def qk_norm_rope_bwd_quantize_fp8(dq, dk, dv, q, k, gamma_q=None, gamma_k=None, rope=None, positions=None, eps=1e-6,
                                  fmt=E4M3, mode=SCALE_TENSOR, rnd=SCALE_FP32, want_q=True, want_qT=False,
                                  want_dgamma=True, out=None, ws=None):
    """qk_norm_rope_bwd with its dqkv quantised (for the QKV projection's Dgrad and Wgrad) instead of written;
    returns dict(q, scale, qT, scaleT, dgamma_q, dgamma_k). Heads of 64 or 128 values."""
    batch, seq, hq, hk, d = sizes = _qk_sizes(dq, dk)
    args = _qk_grads(dq, dk, dv, q, k, gamma_q, gamma_k, rope, positions, eps, sizes, _current())
    q8, scale, qT, scaleT = _quant_outputs(batch * seq, (hq + 2 * hk) * d, mode, want_q, want_qT, out, dq.device)
    dgq, dgk = _dgamma(gamma_q, want_dgamma, d, dq.device), _dgamma(gamma_k, want_dgamma, d, dq.device)
    ws, nb = _ws(_size("puro_qk_norm_rope_bwd_quantize_workspace_size", *sizes), ws, dq.device)
    _check("puro_qk_norm_rope_bwd_quantize_fp8", lib().puro_qk_norm_rope_bwd_quantize_fp8(
        *args, fmt, mode, rnd, _ptr(q8), _ptr(scale), _ptr(qT), _ptr(scaleT), _ptr(dgq), _ptr(dgk), _ptr(ws), nb,
        _stream()))
    return dict(q=q8, scale=scale, qT=qT, scaleT=scaleT, dgamma_q=dgq, dgamma_k=dgk)


def _grad_heads(t):
    """A gradient as the backward takes it: BF16, 16-byte vectors within a head."""
    t = t.to(torch.bfloat16)
    fits = t.stride(-1) == 1 and t.data_ptr() % 16 == 0 and all(s >= 0 and s % 8 == 0 for s in t.stride()[:-1])
    return t if fits else t.contiguous()


class _QkNormRopeFn(torch.autograd.Function):
    """(q, k, v) heads of a QKV projection's output through puro_qk_norm_rope_fwd; the backward assembles the
    gradient of that output in one call from the saved output itself (nothing else is kept)."""

    @staticmethod
    def forward(ctx, qkv, gamma_q, gamma_k, heads_q, heads_k, rope, positions, eps):
        if qkv.dtype != torch.bfloat16:
            raise TypeError("the query / key norm takes BF16 heads")
        heads = qkv.unflatten(-1, (heads_q + 2 * heads_k, -1))
        q, k, v = heads.split((heads_q, heads_k, heads_k), dim=-2)
        ctx.save_for_backward(qkv, gamma_q, gamma_k, positions, rope.table if rope is not None else None)
        ctx.args = heads_q, heads_k, rope is not None and rope.interleaved, eps
        q, k = qk_norm_rope_fwd(q, k, gamma_q, gamma_k, rope, positions, eps)
        return q, k, v

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk, dv):
        qkv, gamma_q, gamma_k, positions, table = ctx.saved_tensors
        heads_q, heads_k, interleaved, eps = ctx.args
        rope = Rope(table, interleaved) if table is not None else None
        q, k, _ = qkv.unflatten(-1, (heads_q + 2 * heads_k, -1)).split((heads_q, heads_k, heads_k), dim=-2)
        dqkv, dgq, dgk = qk_norm_rope_bwd(_grad_heads(dq), _grad_heads(dk), _grad_heads(dv), q, k, gamma_q, gamma_k,
                                          rope, positions, eps, want_dgamma=any(ctx.needs_input_grad[1:3]))
        return (dqkv.view(qkv.shape), dgq.to(gamma_q.dtype) if dgq is not None else None,
                dgk.to(gamma_k.dtype) if dgk is not None else None, None, None, None, None, None)


def qk_norm_rope(qkv, heads_q, heads_k, gamma_q=None, gamma_k=None, rope=None, positions=None, eps=1e-6):
    """The query / key norm with rotation as an autograd operation on a QKV projection's output [.., S, (Hq + 2 Hk) D]
    (BF16, one or no leading batch dimension): returns q [.., S, Hq, D], k and v [.., S, Hk, D] for attention (v is a
    view of qkv)."""
    return _QkNormRopeFn.apply(qkv, gamma_q, gamma_k, heads_q, heads_k, rope, positions, eps)


# ------------------------------------------------------------------- GEMM
def operand(data, fmt, mode, scale):
    """Describe a reduction-contiguous FP8 operand [rows, K]."""
    op = Operand(data.data_ptr(), _ld(data), fmt, mode, scale.data_ptr())
    op._keep = (data, scale)
    return op


def fp8_gemm_workspace_size(M, N, K, out_dtype):
    return _size("puro_fp8_gemm_workspace_size", M, N, K, out_dtype)


def fp8_gemm_plan(M, N, K, a_mode=SCALE_TENSOR, b_mode=SCALE_TENSOR):
    """The plan puro_fp8_gemm takes: dict(tile_m, tile_n, stages, splits, launches)."""
    v = [_i() for _ in range(5)]
    _check("puro_fp8_gemm_plan", lib().puro_fp8_gemm_plan(M, N, K, a_mode, b_mode, *[ctypes.byref(x) for x in v]))
    return dict(zip(("tile_m", "tile_n", "stages", "splits", "launches"), (x.value for x in v)))


def fp8_gemm(A, a_rows, B, b_rows, K, out_dtype=OUT_BF16, D=None, accumulate=False, ws=None):
    """D[M, N] (+)= sum_k A[m, k] B[n, k] with M = a_rows, N = b_rows."""
    M, N = a_rows, b_rows
    dev = torch.device("cuda", torch.cuda.current_device())
    if D is None:
        dt = torch.bfloat16 if out_dtype == OUT_BF16 else torch.float32
        D = torch.empty(M, N, dtype=dt, device=dev)
    w, nb = _ws(fp8_gemm_workspace_size(M, N, K, out_dtype), ws, dev)
    _check("puro_fp8_gemm", lib().puro_fp8_gemm(M, N, K, ctypes.byref(A), ctypes.byref(B), _ptr(D),
                                                out_dtype, _ld(D), int(bool(accumulate)), _ptr(w), nb,
                                                _stream()))
    return D


def fp8_gemm_epilogue(A, a_rows, B, b_rows, K, bias=None, residual=None, D=None, ws=None):
    """D[M, N] = BF16(sum_k A[m, k] B[n, k] + bias[n] + residual[m, n]) (bias
    and residual BF16, optional; residual may be D itself)."""
    M, N = a_rows, b_rows
    dev = torch.device("cuda", torch.cuda.current_device())
    if D is None:
        D = torch.empty(M, N, dtype=torch.bfloat16, device=dev)
    w, nb = _ws(fp8_gemm_workspace_size(M, N, K, OUT_BF16), ws, dev)
    ldr = _ld(residual) if residual is not None else 0
    _check("puro_fp8_gemm_epilogue", lib().puro_fp8_gemm_epilogue(
        M, N, K, ctypes.byref(A), ctypes.byref(B), _ptr(D), _ld(D), _ptr(bias), _ptr(residual), ldr, _ptr(w), nb,
        _stream()))
    return D


# ----------------------------------------------------------- linear layer
@dataclass
class LinearRecipe:
    x_fmt: int = E4M3
    w_fmt: int = E4M3
    dy_fmt: int = E5M2
    blockwise: int = 0
    rnd: int = SCALE_FP32

    def c(self):
        return Recipe(*self.key())

    def key(self):
        return (self.x_fmt, self.w_fmt, self.dy_fmt, self.blockwise, self.rnd)


@functools.lru_cache(maxsize=64, typed=True)
def _recipe_ref(*key):
    """The C recipe of a LinearRecipe's fields, by reference (read only)."""
    return ctypes.byref(Recipe(*key))


@functools.lru_cache(maxsize=1024, typed=True)
def _saved_sizes(M, N, K, *key):
    sizes = (_sz * 4)()
    lib().puro_linear_saved_bytes(M, N, K, _recipe_ref(*key), ctypes.byref(sizes))
    return list(sizes)


@functools.lru_cache(maxsize=1024, typed=True)
def _linear_size(fn, M, N, K, *key):
    return getattr(lib(), fn)(M, N, K, _recipe_ref(*key))


def linear_saved(M, N, K, recipe, device):
    """Allocate the saved-for-backward buffers of a linear layer."""
    G = 128
    xq_t = torch.empty(K, M, dtype=torch.uint8, device=device)
    wq_t = torch.empty(K, N, dtype=torch.uint8, device=device)
    if recipe.blockwise:
        # k-block-major scale layouts (include/puro.h)
        xs = torch.empty(M // G, K, dtype=torch.float32, device=device)
        wsc = torch.empty(N // G, K // G, dtype=torch.float32, device=device)
    else:
        xs = torch.empty(1, dtype=torch.float32, device=device)
        wsc = torch.empty(1, dtype=torch.float32, device=device)
    assert [xq_t.numel(), xs.numel() * 4, wq_t.numel(), wsc.numel() * 4] == _saved_sizes(M, N, K, *recipe.key())
    return dict(xq_t=xq_t, x_scale=xs, wq_t=wq_t, w_scale=wsc)


def _saved_struct(saved):
    return Saved(saved["xq_t"].data_ptr(), saved["x_scale"].data_ptr(), saved["wq_t"].data_ptr(),
                 saved["w_scale"].data_ptr())


def linear_fwd_workspace_size(M, N, K, recipe):
    return _linear_size("puro_linear_fwd_workspace_size", M, N, K, *recipe.key())


def linear_bwd_workspace_size(M, N, K, recipe):
    return _linear_size("puro_linear_bwd_workspace_size", M, N, K, *recipe.key())


def linear_fwd(X, W, recipe, Y=None, saved=None, ws=None):
    """Y = X W^T (FP8 Fprop); returns (Y, saved)."""
    M, K = X.shape
    N = W.shape[0]
    dev = X.device
    if Y is None:
        Y = torch.empty(M, N, dtype=torch.bfloat16, device=dev)
    if saved is None:
        saved = linear_saved(M, N, K, recipe, dev)
    w, nb = _ws(linear_fwd_workspace_size(M, N, K, recipe), ws, dev)
    s = _saved_struct(saved)
    _check("puro_linear_fwd", lib().puro_linear_fwd(_ptr(X), _ptr(W), M, N, K, _recipe_ref(*recipe.key()),
                                                    _ptr(Y), ctypes.byref(s), _ptr(w), nb, _stream()))
    return Y, saved


def linear_bwd(dY, saved, recipe, K, want_dx=True, want_dw=True, dX=None, dW=None, accumulate_dw=False,
               ws=None):
    """dX = dY W (BF16) and dW = dY^T X (FP32); returns (dX, dW)."""
    M, N = dY.shape
    dev = dY.device
    if want_dx and dX is None:
        dX = torch.empty(M, K, dtype=torch.bfloat16, device=dev)
    if want_dw and dW is None:
        dW = torch.zeros(N, K, dtype=torch.float32, device=dev)
    w, nb = _ws(linear_bwd_workspace_size(M, N, K, recipe), ws, dev)
    s = _saved_struct(saved)
    _check("puro_linear_bwd", lib().puro_linear_bwd(
        _ptr(dY), ctypes.byref(s), M, N, K, _recipe_ref(*recipe.key()), _ptr(dX if want_dx else None),
        _ptr(dW if want_dw else None), int(bool(accumulate_dw)), _ptr(w), nb, _stream()))
    return (dX if want_dx else None), (dW if want_dw else None)


class _LinearFn(torch.autograd.Function):
    """Y = X W^T through puro_linear_fwd; the backward runs puro_linear_bwd
    from the FP8 copies the forward saved (the BF16 X is not kept). With a
    ``main_grad`` FP32 buffer on W, dW is accumulated into it by the Wgrad
    GEMM and W gets no .grad; otherwise W's .grad is dW in W's dtype."""

    @staticmethod
    def forward(ctx, X, W, recipe):
        if X.dtype != torch.bfloat16 or W.dtype != torch.bfloat16:
            raise TypeError("the FP8 linear layer takes BF16 X and W")
        Y, saved = linear_fwd(X.contiguous(), W.contiguous(), recipe)
        ctx.saved, ctx.recipe, ctx.K = saved, recipe, X.shape[1]
        ctx.main_grad = getattr(W, "main_grad", None)
        return Y

    @staticmethod
    def backward(ctx, dY):
        want_dx, want_dw = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
        mg = ctx.main_grad if want_dw else None
        dX, dW = linear_bwd(dY.to(torch.bfloat16).contiguous(), ctx.saved, ctx.recipe, ctx.K, want_dx=want_dx,
                            want_dw=want_dw, dW=mg, accumulate_dw=mg is not None)
        ctx.saved = None
        if mg is not None:
            return dX, None, None
        return dX, (dW.to(torch.bfloat16) if dW is not None else None), None


def linear(X, W, recipe):
    """The FP8 linear layer as an autograd operation: X [..., K], W [N, K]
    (BF16); returns Y [..., N] (BF16)."""
    shp = X.shape
    Y = _LinearFn.apply(X.reshape(-1, shp[-1]), W, recipe)
    return Y.reshape(*shp[:-1], Y.shape[-1])


class Linear(torch.nn.Module):
    """A bias-free linear layer whose forward and backward run the FP8 path
    (default: the paper's blockwise recipe, E4M3 with power-of-two scales).
    The weight is BF16, as the model's GEMM operands are (Appendix C); with
    ``main_grad`` (default) its FP32 gradient is accumulated into
    ``weight.main_grad`` across backward passes, for an optimiser that keeps
    FP32 state (zero it after each step)."""

    def __init__(self, in_features, out_features, recipe=None, main_grad=True, device=None):
        super().__init__()
        self.in_features, self.out_features = in_features, out_features
        self.recipe = recipe if recipe is not None else LinearRecipe(E4M3, E4M3, E4M3, 1, SCALE_POW2)
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, dtype=torch.bfloat16,
                                                     device=device))
        with torch.no_grad():
            self.weight.normal_(0.0, 0.02)
        if main_grad:
            self.weight.main_grad = torch.zeros(out_features, in_features, dtype=torch.float32,
                                                device=self.weight.device)

    def forward(self, x):
        return linear(x, self.weight, self.recipe)


# ------------------------------------------ LM head with cross-entropy loss
LM_HEAD_BF16, LM_HEAD_FP8 = 0, 1


def lm_head_ce_workspace_size(M, V, K, recipe, backward):
    return lib().puro_lm_head_ce_workspace_size(M, V, K, recipe, int(bool(backward)))


def lm_head_ce_fwd(X, W, targets, recipe=LM_HEAD_BF16, lse=None, loss=None, ws=None):
    """lse [M] and loss [M] = lse - z_target of the logits X W^T (never
    stored); X [M, K], W [V, K] BF16, targets [M] int32; returns (lse, loss)."""
    M, K = X.shape
    V = W.shape[0]
    dev = X.device
    lse = torch.empty(M, dtype=torch.float32, device=dev) if lse is None else lse
    loss = torch.empty(M, dtype=torch.float32, device=dev) if loss is None else loss
    w, nb = _ws(lm_head_ce_workspace_size(M, V, K, recipe, False), ws, dev)
    _check("puro_lm_head_ce_fwd", lib().puro_lm_head_ce_fwd(
        _ptr(X), _ptr(W), _ptr(targets), M, V, K, recipe, _ptr(lse), _ptr(loss), _ptr(w), nb, _stream()))
    return lse, loss


def lm_head_ce_bwd(X, W, targets, lse, recipe=LM_HEAD_BF16, grad_scale=1.0, dX=None, dW=None, ws=None):
    """dX [M, K] (BF16) and dW [V, K] (FP32) of grad_scale * sum of the losses."""
    M, K = X.shape
    V = W.shape[0]
    dev = X.device
    dX = torch.empty(M, K, dtype=torch.bfloat16, device=dev) if dX is None else dX
    dW = torch.empty(V, K, dtype=torch.float32, device=dev) if dW is None else dW
    w, nb = _ws(lm_head_ce_workspace_size(M, V, K, recipe, True), ws, dev)
    _check("puro_lm_head_ce_bwd", lib().puro_lm_head_ce_bwd(
        _ptr(X), _ptr(W), _ptr(targets), _ptr(lse), M, V, K, recipe, float(grad_scale), _ptr(dX), _ptr(dW),
        _ptr(w), nb, _stream()))
    return dX, dW


# ------------------------------------- LM head with a teacher's top logits
DISTILL_LOGITS, DISTILL_PROBS = 0, 1


def lm_head_distill_workspace_size(M, V, K, topk, backward):
    return _size("puro_lm_head_distill_workspace_size", M, V, K, topk, int(bool(backward)))


def _dense(t, what, dtypes, shape, device):
    if t.dtype not in dtypes or t.get_device() != device:
        _check_tensor(t, what, dtypes, device)
    if t.shape != shape or not t.is_contiguous():
        raise ValueError("%s: a contiguous %s tensor expected, got %s" % (what, shape, tuple(t.shape)))
    return t.data_ptr()


def _distill_args(X, W, ids, teacher, dev):
    """Sizes and the pointers of the inputs that both passes take."""
    x, w, i = X.shape, W.shape, ids.shape
    if len(x) != 2 or len(w) != 2 or len(i) != 2:
        raise ValueError("X [M, K], W [V, K], ids and teacher [M, topk]")
    (M, K), V, k = x, w[0], i[1]
    return M, V, K, k, (_dense(X, "X", _BF16_BITS, (M, K), dev), _dense(W, "W", _BF16_BITS, (V, K), dev),
                        _dense(ids, "ids", _INT32, (M, k), dev), _dense(teacher, "teacher", _FP32, (M, k), dev))


def lm_head_distill_fwd(X, W, ids, teacher, temperature=1.0, target=DISTILL_LOGITS, lse=None, loss=None, z_top=None,
                        ws=None):
    """The divergence of softmax(X W^T / temperature) from a teacher known by its topk entries per row: ids [M, topk]
    int32 (-1: none) and teacher [M, topk] FP32 logits (their softmax is taken) or probabilities (DISTILL_PROBS).
    Returns (lse, loss, z_top): [M], [M] and the student's logits [M, topk]; the logits X W^T are never stored."""
    dev = _current()
    M, V, K, k, inputs = _distill_args(X, W, ids, teacher, dev)
    lse, loss, z_top = (teacher.new_empty(*shape) if t is None else t
                        for t, shape in ((lse, (M,)), (loss, (M,)), (z_top, (M, k))))
    w, nb = _ws(lm_head_distill_workspace_size(M, V, K, k, False), ws, X.device)
    _check("puro_lm_head_distill_fwd", lib().puro_lm_head_distill_fwd(
        *inputs, M, V, K, k, target, temperature, _dense(lse, "lse", _FP32, (M,), dev), _dense(loss, "loss", _FP32, (M,), dev),
        _dense(z_top, "z_top", _FP32, (M, k), dev), _ptr(w), nb, _stream()))
    return lse, loss, z_top


def lm_head_distill_bwd(X, W, ids, teacher, lse, z_top, temperature=1.0, target=DISTILL_LOGITS, dloss=None,
                        grad_scale=1.0, want_dx=True, want_dw=True, dX=None, dW=None, accumulate_dw=False, ws=None):
    """dX [M, K] (BF16) and dW [V, K] (FP32; a BF16 tensor given as dW is filled in BF16) of grad_scale times the sum
    of dloss [M] (None: ones) times the losses, from what the forward kept."""
    dev = _current()
    M, V, K, k, inputs = _distill_args(X, W, ids, teacher, dev)
    if want_dx and dX is None:
        dX = torch.empty(M, K, dtype=torch.bfloat16, device=X.device)
    if want_dw and dW is None:
        dW = (torch.zeros if accumulate_dw else torch.empty)(V, K, dtype=torch.float32, device=X.device)
    px = _dense(dX, "dX", _BF16_BITS, (M, K), dev) if want_dx else None
    pw = _dense(dW, "dW", (torch.float32, torch.bfloat16), (V, K), dev) if want_dw else None
    out = OUT_BF16 if want_dw and dW.dtype == torch.bfloat16 else OUT_FP32
    w, nb = _ws(lm_head_distill_workspace_size(M, V, K, k, True), ws, X.device)
    _check("puro_lm_head_distill_bwd", lib().puro_lm_head_distill_bwd(
        *inputs, _dense(lse, "lse", _FP32, (M,), dev), _dense(z_top, "z_top", _FP32, (M, k), dev), M, V, K, k, target,
        temperature, _dense(dloss, "dloss", _FP32, (M,), dev) if dloss is not None else None, grad_scale, px, pw, out,
        int(bool(accumulate_dw)), _ptr(w), nb, _stream()))
    return (dX if want_dx else None), (dW if want_dw else None)


class _DistillFn(torch.autograd.Function):
    """loss [M] through puro_lm_head_distill_fwd; the backward recomputes the logits. With a ``main_grad`` FP32
    buffer on W, dW is accumulated into it and W gets no .grad; otherwise W's .grad is dW in BF16."""

    @staticmethod
    def forward(ctx, X, W, ids, teacher, temperature, target):
        if X.dtype != torch.bfloat16 or W.dtype != torch.bfloat16:
            raise TypeError("the LM head takes BF16 X and W")
        main_grad = getattr(W, "main_grad", None)
        X, W = X.contiguous(), W.contiguous()
        lse, loss, z_top = lm_head_distill_fwd(X, W, ids, teacher, temperature, target)
        ctx.save_for_backward(X, W, ids, teacher, lse, z_top)
        ctx.args = temperature, target, main_grad
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        X, W, ids, teacher, lse, z_top = ctx.saved_tensors
        temperature, target, mg = ctx.args
        want_dx, want_dw = ctx.needs_input_grad[:2]
        dW = mg if mg is not None or not want_dw else torch.empty_like(W)
        dX, dW = lm_head_distill_bwd(X, W, ids, teacher, lse, z_top, temperature, target, dloss.contiguous(),
                                     want_dx=want_dx, want_dw=want_dw, dW=dW, accumulate_dw=want_dw and mg is not None)
        return dX, dW if mg is None else None, None, None, None, None


def lm_head_distill(X, W, ids, teacher, temperature=1.0, target=DISTILL_LOGITS):
    """The distillation loss [M] of X [M, K] and W [V, K] (BF16) as an autograd operation (``lm_head_distill_fwd``);
    no gradient flows to the teacher's values."""
    return _DistillFn.apply(X, W, ids, teacher, temperature, target)


# -------------------------------------------- 8-bit integer linear layers
# (calls of few microseconds: as few checks each as keep a kernel from foreign memory)
_INT8 = (torch.int8,)


def _matrix(t, what, dtypes, device):
    """(rows, cols, row pitch, address) of a 2-D tensor with contiguous rows."""
    if t.dtype not in dtypes or t.get_device() != device:
        _check_tensor(t, what, dtypes, device)
    if t.dim() != 2:
        raise ValueError("%s: 2-D expected, got %s" % (what, tuple(t.shape)))
    rows, cols = t.shape
    ld, one = t.stride()
    if rows <= 1 or cols <= 1:
        if one != 1 and cols > 1 and rows > 0:
            raise ValueError("%s: the values of a row are contiguous" % what)
        if rows <= 1 or cols == 0:
            ld = -(-cols // 16) * 16           # (the pitch of one row, or of none, is any)
    elif one != 1:
        raise ValueError("%s: the values of a row are contiguous" % what)
    return rows, cols, ld, t.data_ptr()


def _vector(t, what, dtypes, n, device):
    if t.dtype not in dtypes or t.get_device() != device:
        _check_tensor(t, what, dtypes, device)
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError("%s: %d contiguous values expected, got %s" % (what, n, tuple(t.shape)))
    return t.data_ptr()


def _int8_rows(rows, cols, out, like, dev):
    """q [rows, cols] and scale [rows], given or new, and their addresses."""
    q = scale = None
    if out:
        q, scale = out.get("q"), out.get("scale")
    if q is None:
        q = like.new_empty((rows, cols), dtype=torch.int8)
    else:
        _dense(q, "q", _INT8, (rows, cols), dev)
    if scale is None:
        scale = like.new_empty(rows, dtype=torch.float32)
    else:
        _vector(scale, "scale", _FP32, rows, dev)
    return q, scale, q.data_ptr(), scale.data_ptr()


def quantize_int8(x, want_q=True, want_qT=False, out=None, ws=None):
    """int8 codes of a BF16 tensor [rows, cols]: q [rows, cols] with scale [rows] (a token's, or an output channel's of a
    weight) and, with want_qT, the transposed copy qT [cols, rows rounded up to 16] (zeros behind the rows) with scaleT
    [cols]; returns dict(q, scale, qT, scaleT) (absent outputs are None). ``out`` may supply outputs; a given qT may have
    a longer pitch."""
    dev = _current()
    rows, cols, ld, px = _matrix(x, "x", _BF16_BITS, dev)
    q = scale = qT = scaleT = pq = ps = pT = psT = None
    nb, ldT = 0, -(-rows // 16) * 16
    if want_q:
        q, scale, pq, ps = _int8_rows(rows, cols, out, x, dev)
    if want_qT:
        qT, scaleT = (out or {}).get("qT"), (out or {}).get("scaleT")
        qT = x.new_empty((cols, ldT), dtype=torch.int8) if qT is None else qT
        scaleT = x.new_empty(cols, dtype=torch.float32) if scaleT is None else scaleT
        if qT.shape != (cols, ldT):
            raise ValueError("qT: shape %s expected, got %s" % ((cols, ldT), tuple(qT.shape)))
        _, _, ldT, pT = _matrix(qT, "qT", _INT8, dev)
        psT = _vector(scaleT, "scaleT", _FP32, cols, dev)
        ws, nb = _ws(_size("puro_quantize_int8_workspace_size", rows, cols), ws, x.device)
    if rows == 0 or cols == 0:                 # (sums of nothing are scaled by these)
        for s in (scale, scaleT):
            if s is not None:
                s.fill_(1.0)
    _check("puro_quantize_int8", lib().puro_quantize_int8(px, rows, cols, ld, pq, ps, pT, ldT, psT, _ptr(ws) if nb else None, nb,
                                                          _stream()))
    return dict(q=q, scale=scale, qT=qT, scaleT=scaleT)


def rmsnorm_quantize_int8(x, gamma, eps, want_rstd=False, out=None):
    """int8 codes of y = x rstd gamma (RMSNorm of each row of x) with a scale per row, y not written (nor rounded to
    BF16); returns dict(q, scale, rstd), rstd [rows] FP32 if it is wanted."""
    dev = _current()
    rows, cols, ld, px = _matrix(x, "x", _BF16_BITS, dev)
    q, scale, pq, ps = _int8_rows(rows, cols, out, x, dev)
    rstd = out.get("rstd") if out else None
    if rstd is None and want_rstd:
        rstd = x.new_empty(rows, dtype=torch.float32)
    _check("puro_rmsnorm_quantize_int8", lib().puro_rmsnorm_quantize_int8(
        px, _vector(gamma, "gamma", _BF16_BITS, cols, dev), rows, cols, ld, eps, pq, ps,
        _vector(rstd, "rstd", _FP32, rows, dev) if rstd is not None else None, _stream()))
    return dict(q=q, scale=scale, rstd=rstd)


def swiglu_quantize_int8(gu, cols, out=None):
    """int8 codes of H = silu(gate) up of a fused gate/up output gu [rows, 2 cols] with a scale per row, H not written
    (nor rounded to BF16); returns dict(q, scale)."""
    dev = _current()
    rows, width, ld, px = _matrix(gu, "gu", _BF16_BITS, dev)
    if width < 2 * cols:
        raise ValueError("gu: %d columns for two halves of %d" % (width, cols))
    q, scale, pq, ps = _int8_rows(rows, cols, out, gu, dev)
    if cols == 0:                              # (as quantize_int8)
        scale.fill_(1.0)
    _check("puro_swiglu_quantize_int8", lib().puro_swiglu_quantize_int8(px, rows, cols, ld, pq, ps, _stream()))
    return dict(q=q, scale=scale)


def int8_gemm(A, a_scale, B, b_scale, out_dtype=OUT_BF16, D=None, accumulate=False, bias=None, residual=None, ws=None):
    """D[M, N] (+)= (sum_k A[m, k] B[n, k]) a_scale[m] b_scale[n] (+ bias[n] + residual[m, n]) of int8 codes A [M, K] and
    B [N, K]; D BF16 or FP32 (its own type, if given); accumulate with FP32, bias and residual (BF16) with BF16."""
    dev = _current()
    M, K, lda, pa = _matrix(A, "A", _INT8, dev)
    N, K_b, ldb, pb = _matrix(B, "B", _INT8, dev)
    if K != K_b:
        raise ValueError("A %s and B %s differ in their columns" % (tuple(A.shape), tuple(B.shape)))
    if D is None:
        if out_dtype not in (OUT_BF16, OUT_FP32):
            raise ValueError("out_dtype is OUT_BF16 or OUT_FP32")
        ldd = -(-N // 4) * 4
        D = (torch.zeros if accumulate else torch.empty)(M, ldd, dtype=torch.float32 if out_dtype == OUT_FP32 else torch.bfloat16,
                                                         device=A.device)
        D = D if ldd == N else D[:, :N]
        pd = D.data_ptr()
    else:
        if D.shape != (M, N):
            raise ValueError("D: shape %s expected, got %s" % ((M, N), tuple(D.shape)))
        _, _, ldd, pd = _matrix(D, "D", (torch.bfloat16, torch.float32), dev)
    ldr, pr = 0, None
    if residual is not None:
        if residual.shape != (M, N):
            raise ValueError("residual: shape %s expected, got %s" % ((M, N), tuple(residual.shape)))
        _, _, ldr, pr = _matrix(residual, "residual", _BF16_BITS, dev)
    w, nb = _ws(_size("puro_int8_gemm_workspace_size", M, N, K), ws, A.device)
    _check("puro_int8_gemm", lib().puro_int8_gemm(
        M, N, K, pa, lda, _vector(a_scale, "a_scale", _FP32, M, dev), pb, ldb, _vector(b_scale, "b_scale", _FP32, N, dev), pd,
        OUT_FP32 if D.dtype == torch.float32 else OUT_BF16, ldd, int(bool(accumulate)),
        _vector(bias, "bias", _BF16_BITS, N, dev) if bias is not None else None, pr, ldr, _ptr(w), nb, _stream()))
    return D


def int8_linear_fwd(X, W, Y=None, want_saved=True, ws=None, want_dx=True, want_dw=True):
    """Y = X W^T [M, N] (BF16) of BF16 X [M, K] and W [N, K], both quantised to int8, a scale per token and per output
    channel; returns (Y, saved): the transposed copies with scales per channel that ``int8_linear_bwd`` takes (None
    without want_saved), W's for dX and X's for dW, None where that gradient will not be wanted."""
    dev = _current()
    (M, K), N = X.shape, W.shape[0]
    px, pw = _dense(X, "X", _BF16_BITS, (M, K), dev), _dense(W, "W", _BF16_BITS, (N, K), dev)
    if Y is None:
        Y = X.new_empty((M, N), dtype=torch.bfloat16)
    saved = s = None
    if want_saved:
        saved = dict(xq_t=X.new_empty((K, -(-M // 16) * 16), dtype=torch.int8) if want_dw else None,
                     x_scale=X.new_empty(K, dtype=torch.float32) if want_dw else None,
                     wq_t=X.new_empty((K, N), dtype=torch.int8) if want_dx else None,
                     w_scale=X.new_empty(K, dtype=torch.float32) if want_dx else None)
        s = ctypes.byref(Saved(*map(_ptr, saved.values())))
    w, nb = _ws(_size("puro_int8_linear_fwd_workspace_size", M, N, K), ws, X.device)
    _check("puro_int8_linear_fwd", lib().puro_int8_linear_fwd(
        px, pw, M, N, K, _dense(Y, "Y", (torch.bfloat16,), (M, N), dev), s, _ptr(w), nb, _stream()))
    return Y, saved


def int8_linear_bwd(dY, saved, want_dx=True, want_dw=True, dX=None, dW=None, accumulate_dw=False, ws=None):
    """dX = dY W [M, K] (BF16) and dW = dY^T X [N, K] (FP32) with dY [M, N] (BF16) quantised to int8 per token for the one
    and per channel for the other; returns (dX, dW)."""
    dev = _current()
    (M, N), xq, wq = dY.shape, saved["xq_t"], saved["wq_t"]
    if (want_dw and xq is None) or (want_dx and wq is None):
        raise ValueError("the forward did not save what %s is made of" % ("dW" if want_dw and xq is None else "dX"))
    K = (wq if xq is None else xq).shape[0] if xq is not None or wq is not None else 0
    pdy = _dense(dY, "dY", _BF16_BITS, (M, N), dev)
    s = Saved(None, None, None, None)
    if xq is not None:
        s.xq_t, s.x_scale = _dense(xq, "xq_t", _INT8, (K, -(-M // 16) * 16), dev), _vector(saved["x_scale"], "x_scale", _FP32, K, dev)
    if wq is not None:
        s.wq_t, s.w_scale = _dense(wq, "wq_t", _INT8, (K, N), dev), _vector(saved["w_scale"], "w_scale", _FP32, K, dev)
    pdx = pdw = None
    if want_dx:
        if dX is None:
            dX = dY.new_empty((M, K), dtype=torch.bfloat16)
        pdx = _dense(dX, "dX", (torch.bfloat16,), (M, K), dev)
    if want_dw:
        if dW is None:
            dW = (dY.new_zeros if accumulate_dw else dY.new_empty)((N, K), dtype=torch.float32)
        pdw = _dense(dW, "dW", _FP32, (N, K), dev)
    w, nb = _ws(_size("puro_int8_linear_bwd_workspace_size", M, N, K), ws, dY.device)
    _check("puro_int8_linear_bwd", lib().puro_int8_linear_bwd(
        pdy, ctypes.byref(s), M, N, K, pdx, pdw, int(bool(accumulate_dw)), _ptr(w), nb, _stream()))
    return (dX if want_dx else None), (dW if want_dw else None)


def _dense_rows(t):
    """A tensor as the int8 linear layer takes it: contiguous, 16-byte aligned."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class _Int8LinearFn(torch.autograd.Function):
    """Y = X W^T through int8_linear_fwd; the backward takes the rounding's derivative as 1. With a ``main_grad`` FP32
    buffer on W, dW is accumulated into it and W gets no .grad; otherwise W's .grad is dW in W's dtype."""

    @staticmethod
    def forward(ctx, X, W, keep):
        want_dx, want_dw, _ = ctx.needs_input_grad
        Y, saved = int8_linear_fwd(_dense_rows(X), _dense_rows(W), want_saved=keep, want_dx=want_dx, want_dw=want_dw)
        if keep:
            ctx.save_for_backward(*saved.values())
            ctx.main_grad = getattr(W, "main_grad", None)
        return Y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dY):
        saved = dict(zip(("xq_t", "x_scale", "wq_t", "w_scale"), ctx.saved_tensors))
        want_dx, want_dw, _ = ctx.needs_input_grad
        mg = ctx.main_grad if want_dw else None
        dX, dW = int8_linear_bwd(_dense_rows(dY.to(torch.bfloat16)), saved, want_dx, want_dw, dW=mg, accumulate_dw=mg is not None)
        return dX, dW.to(torch.bfloat16) if want_dw and mg is None else None, None


def int8_linear(X, W):
    """The int8 linear layer as an autograd operation: X [..., K], W [N, K] (BF16); returns Y [..., N] (BF16). N and K are
    multiples of 16, the number of tokens is any."""
    if X.dtype != torch.bfloat16 or W.dtype != torch.bfloat16:
        raise TypeError("the int8 linear layer takes BF16 X and W")
    rows = X.reshape(X.shape[:-1].numel(), X.shape[-1])
    keep = torch.is_grad_enabled() and (X.requires_grad or W.requires_grad)
    # (a tangent of forward mode is refused there, rather than lost)
    if keep or any(torch.autograd.forward_ad.unpack_dual(t).tangent is not None for t in (X, W)):
        Y = _Int8LinearFn.apply(rows, W, keep)
    else:
        Y, _ = int8_linear_fwd(_dense_rows(rows.detach()), _dense_rows(W.detach()), want_saved=False)
    return Y.reshape(*X.shape[:-1], Y.shape[-1])


# ----------------------------------------- verification of drafted tokens
VERIFY_LOGITS, VERIFY_PROBS = 0, 1


def verify_drafts(target, draft, draft_ids, offsets, uniform=None, uniform_sample=None, temperature=1.0, kind=VERIFY_LOGITS,
                  tokens=None, accepted=None, ws=None):
    """Which drafted tokens to keep, and the token after them. target [T, V] (BF16 or FP32): the rows of all sequences one
    after another, sequence b's from offsets[b] to offsets[b + 1] (int32 [B + 1]), one more than it has drafts (or none: an
    idle slot); draft [drafts, V] of target's type: the draft model's predictions, a row for each draft, sequence by
    sequence, None where it has none; draft_ids [T] int32, the last of a sequence not read. Logits, at a temperature (0: the largest), or probabilities
    (VERIFY_PROBS). uniform [T] and uniform_sample [B]: FP32 random numbers in [0, 1). Returns (tokens [T], accepted [B])
    int32: a sequence's kept ids, its drawn token and -1 from there on; rows behind the last sequence are left alone."""
    dev = _current()
    T, V, ldt, pt = _matrix(target, "target", (torch.bfloat16, torch.float32), dev)
    if offsets.dim() != 1 or offsets.shape[0] == 0:
        raise ValueError("offsets: one more than there are sequences")
    B = offsets.shape[0] - 1
    rows, ldd, pd = 0, 0, None
    if draft is not None:
        rows, V_d, ldd, pd = _matrix(draft, "draft", (target.dtype,), dev)
        if V_d != V:
            raise ValueError("target %s and draft %s differ in their columns" % (tuple(target.shape), tuple(draft.shape)))
        pd = pd or pt                          # (no rows have no address; none is read)
    pids = _vector(draft_ids, "draft_ids", _INT32, T, dev)
    if tokens is None:
        tokens = draft_ids.new_empty(T)
    else:
        _vector(tokens, "tokens", _INT32, T, dev)
    if accepted is None:
        accepted = draft_ids.new_empty(B)
    else:
        _vector(accepted, "accepted", _INT32, B, dev)
    w, nb = _ws(_size("puro_verify_drafts_workspace_size", B, T, rows, V), ws, target.device)
    _check("puro_verify_drafts", lib().puro_verify_drafts(
        B, T, rows, V, kind, OUT_BF16 if target.dtype == torch.bfloat16 else OUT_FP32, pt, ldt, pd, ldd,
        pids, _vector(offsets, "offsets", _INT32, B + 1, dev),
        _vector(uniform, "uniform", _FP32, T, dev) if uniform is not None else None,
        _vector(uniform_sample, "uniform_sample", _FP32, B, dev) if uniform_sample is not None else None, temperature,
        tokens.data_ptr(), accepted.data_ptr(), _ptr(w), nb, _stream()))
    return tokens, accepted


# ------------------------------------------------------------------- MuonH
def muonh_step(W, G, buf, radius, eta, mu=0.95, nesterov=True, ns_steps=5, w_bf16=None, u_out=None, ws=None):
    """One MuonH step of W [count, rows, cols] (or [rows, cols]) in place,
    with buf (the momentum) updated in place; radius [count] FP32. Returns
    (w_bf16, u_out) when asked for."""
    shp = W.shape
    count, rows, cols = (1,) + tuple(shp) if W.dim() == 2 else tuple(shp)
    w, nb = _ws(lib().puro_muonh_workspace_size(count, rows, cols), ws, W.device)
    _check("puro_muonh_step", lib().puro_muonh_step(
        count, rows, cols, _ptr(W), _ptr(w_bf16), _ptr(G), _ptr(buf), _ptr(radius), float(mu), int(bool(nesterov)),
        float(eta), int(ns_steps), _ptr(u_out), _ptr(w), nb, _stream()))
    return w_bf16, u_out


def newton_schulz_bf16(X, steps=5, out=None, ws=None):
    """steps Newton-Schulz steps on X [count, r, c] (or [r, c]) BF16, r <= c."""
    count, r, c = (1,) + tuple(X.shape) if X.dim() == 2 else tuple(X.shape)
    out = torch.empty_like(X) if out is None else out
    w, nb = _ws(lib().puro_newton_schulz_workspace_size(count, r, c), ws, X.device)
    _check("puro_newton_schulz_bf16", lib().puro_newton_schulz_bf16(
        count, r, c, _ptr(X), int(steps), _ptr(out), _ptr(w), nb, _stream()))
    return out

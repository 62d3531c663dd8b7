"""ctypes binding of libefq_attn.so (argument marshalling only).

Every computation runs in the HIP kernels of ``csrc/efq_attn.hip`` and
``csrc/efq_paged.hip``; torch provides device memory and the current stream.  The functions mirror the C
entry points of ``include/efq_attn.h``.  If the library is missing this
module raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libefq_attn.so")

PGEN_EFQ, PGEN_EXPQ, PGEN_LUT, PGEN_NOOP, PGEN_EXPQ6 = 0, 1, 2, 3, 4
KINDS = {"efq": PGEN_EFQ, "expq": PGEN_EXPQ, "lut": PGEN_LUT, "noop": PGEN_NOOP,
         "expq6": PGEN_EXPQ6}

# (tau, h) operating points of Sec. IV-A, and the LUT constants of Sec. II-D
PARAMS_MEAN = (-3.06, 2.30)
PARAMS_MMLU = (-2.90, 2.00)
PARAMS_BALANCE = (-2.10, 2.70)
PARAMS_LUT = (-3.17805383, 4.40521173)

EFQ_OK, EFQ_EINVAL, EFQ_EUNSUPPORTED, EFQ_EWORKSPACE, EFQ_EHIP = 0, -1, -2, -3, -4


class EfqError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"efq status {status}: {msg}")
        self.status = status


class Shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int), ("seq_q", ctypes.c_int), ("seq_k", ctypes.c_int),
                ("heads_q", ctypes.c_int), ("heads_kv", ctypes.c_int), ("head_dim", ctypes.c_int)]


class Params(ctypes.Structure):
    _fields_ = [("tau", ctypes.c_float), ("h", ctypes.c_float)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class Rotary(ctypes.Structure):
    _fields_ = [("pairs", ctypes.c_int), ("axes", ctypes.c_int), ("interleaved", ctypes.c_int),
                ("inv_freq", ctypes.c_void_p), ("axis", ctypes.c_void_p), ("pos", ctypes.c_void_p)]


class Cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int), ("page_size", ctypes.c_int), ("heads_kv", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("format", ctypes.c_int), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class Batch(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_int), ("tokens", ctypes.c_int), ("table_width", ctypes.c_int),
                ("max_q", ctypes.c_int), ("max_k", ctypes.c_int), ("q_start", ctypes.c_void_p),
                ("seq_k", ctypes.c_void_p), ("page_table", ctypes.c_void_p)]


_lib = None
P = ctypes.c_void_p
SZ = ctypes.c_size_t
I = ctypes.c_int
F = ctypes.c_float
SP = ctypes.POINTER(Shape)
RP, TP, CP, BP = (ctypes.POINTER(t) for t in (Rows, Rotary, Cache, Batch))

SIGNATURES = {
    "efq_abi_version": ([], I),
    "efq_strerror": ([I], ctypes.c_char_p),
    "efq_vhat_bytes": ([SP], SZ),
    "efq_vhat_scale_offset": ([SP], SZ),
    "efq_attn_workspace_bytes": ([SP], SZ),
    "efq_quant_v_mxfp4": ([P, SP, P, SZ, P], I),
    "efq_attn_fwd_vhat": ([P, P, P, SZ, F, I, I, Params, P, SP, P], I),
    "efq_attn_split_bytes": ([SP, I], SZ),
    "efq_attn_fwd_vhat_ws": ([P, P, P, SZ, F, I, I, Params, P, SP, P, SZ, P], I),
    "efq_attn_fwd_ex": ([P, P, P, F, I, I, Params, P, SP, P, SZ, P], I),
    "efq_attn_fwd": ([P, P, P, F, I, P, SP, P], I),
    "efq_attn_fwd_noalloc": ([P, P, P, F, I, I, Params, P, SP, P], I),
    "efq_attn_fwd_expq": ([P, P, P, F, I, P, SP, P], I),
    "efq_pgen": ([P, I, I, I, Params, P, P, P], I),
    "efq_attn_fwd_dump": ([P, P, P, SZ, F, I, I, Params, P, SP, P, P, P, P, P], I),
    "efq_pgen_bench": ([I, Params, I, I, P, P], I),
    "efq_clock_probe": ([I, I, P, P], I),
    "efq_calibrate_workspace_bytes": ([SP, I], SZ),
    "efq_calibrate": ([P, P, P, F, I, P, SP, P, I, P, I, P, ctypes.POINTER(Params), P, SZ, P], I),
    "efq_qhat_bytes": ([SP], SZ),
    "efq_qhat_scale_offset": ([SP], SZ),
    "efq_khat_bytes": ([SP], SZ),
    "efq_khat_scale_offset": ([SP], SZ),
    "efq_quant_qk_mxfp8": ([P, P, SP, P, SZ, P, SZ, P], I),
    "efq_attn_fwd_qk8": ([P, SZ, P, SZ, P, SZ, F, I, I, Params, P, SP, P], I),
    "efq_attn_fwd_qk8_ws": ([P, SZ, P, SZ, P, SZ, F, I, I, Params, P, SP, P, SZ, P], I),
    "efq_attn_fwd_qk8_dump": ([P, SZ, P, SZ, P, SZ, F, I, I, Params, P, SP, P, P, P, P, P], I),
    "efq_attn_lowbit_workspace_bytes": ([SP], SZ),
    "efq_attn_fwd_lowbit_ex": ([P, P, P, F, I, I, Params, P, SP, P, SZ, P], I),
    "efq_rope": ([RP, RP, I, I, I, I, TP, I, P], I),
    "efq_kv_append": ([RP, RP, CP, BP, TP, RP, I, RP, P], I),
    "efq_attn_paged_workspace_bytes": ([CP, BP, I], SZ),
    "efq_attn_paged": ([RP, I, CP, BP, F, I, RP, I, P, P, SZ, P], I),
}


def lib():
    """Load the HIP library (build it first with ``__graft_entry__.build()``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build the HIP library first")
        L = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in SIGNATURES.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        _lib = L
    return _lib


def _check(status: int):
    if status != EFQ_OK:
        raise EfqError(status, lib().efq_strerror(status).decode())


def _stream(stream=None):
    if stream is None:
        # the handle itself: building a Stream object costs 3 us a call
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return ctypes.c_void_p(stream.cuda_stream)


def _ptr(t: Optional[torch.Tensor]):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


def shape_of(q: torch.Tensor, k: torch.Tensor) -> Shape:
    B, Sq, Hq, D = q.shape
    Bk, Sk, Hkv, Dk = k.shape
    if B != Bk or D != Dk:
        raise ValueError("q and k shapes disagree")
    return Shape(B, Sq, Sk, Hq, Hkv, D)


def _params(kind: int, params) -> Params:
    if params is None:
        params = PARAMS_LUT if kind == PGEN_LUT else PARAMS_MEAN
    return Params(float(params[0]), float(params[1]))


def _kind(kind) -> int:
    return KINDS[kind] if isinstance(kind, str) else int(kind)


def _bf16(t: torch.Tensor, name: str):
    if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous bf16 CUDA tensor")


def _scratch(nbytes: int, stream=None) -> Optional[torch.Tensor]:
    """Scratch of one call from torch's allocator, in the memory pool of the
    stream that uses it (so it is reused only after that work), or None.  A
    call without a stream runs on the current device's current stream, whatever
    device its tensors are on; a stream that is only a handle (not torch's) has
    no pool, and gets None."""
    if nbytes == 0 or not (stream is None or isinstance(stream, torch.cuda.Stream)):
        return None
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device="cuda")


def _output(shape, dtype, device, stream=None) -> torch.Tensor:
    """An output that the caller did not bring, in the memory pool of the stream
    the call runs on: a block of the current stream's may be one that its queued
    work still uses.  It is kept, once dropped, until the current stream is
    done with it too, where its reader is most likely to be."""
    if stream is None or stream.cuda_stream == torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()):
        return torch.empty(shape, dtype=dtype, device=device)
    now = torch.cuda.current_stream()
    if not isinstance(stream, torch.cuda.Stream):        # a handle
        stream = torch.cuda.ExternalStream(stream.cuda_stream)
    with torch.cuda.stream(stream):
        out = torch.empty(shape, dtype=dtype, device=device)
    out.record_stream(now)
    return out


def _splits(causal, kind) -> bool:
    """Whether calls of this form may run split over the keys at all."""
    return not causal and kind != PGEN_NOOP


def _workspace(sh: Shape, causal, kind, qk8: bool, workspace, stream):
    """(workspace tensor or None, its bytes) of a whole call.  The caller's, or
    one from torch's allocator, which keeps freed blocks: the library's own
    stream-ordered allocation maps and unmaps device memory on every call."""
    if workspace is None:
        s, l = ctypes.byref(sh), lib()
        if _splits(causal, kind):
            n = l.efq_attn_lowbit_workspace_bytes(s) if qk8 else l.efq_attn_workspace_bytes(s)
        else:
            n = l.efq_vhat_bytes(s) + (l.efq_qhat_bytes(s) + l.efq_khat_bytes(s) if qk8 else 0)
        try:
            workspace = _scratch(int(n), stream)
        except torch.OutOfMemoryError:
            workspace = None            # the library then tries an allocation of its own
    return workspace, 0 if workspace is None else workspace.numel() * workspace.element_size()


def _split_scratch(shape: Shape, causal, kind, qk8: bool, stream):
    """(scratch or None, bytes) of the key split that few queries run by."""
    n = int(lib().efq_attn_split_bytes(ctypes.byref(shape), int(qk8))) if _splits(causal, kind) else 0
    try:
        scratch = _scratch(n, stream)
    except torch.OutOfMemoryError:      # without scratch the unsplit kernels run
        scratch = None
    return scratch, 0 if scratch is None else n


def vhat_bytes(shape: Shape) -> int:
    return int(lib().efq_vhat_bytes(ctypes.byref(shape)))


def vhat_scale_offset(shape: Shape) -> int:
    return int(lib().efq_vhat_scale_offset(ctypes.byref(shape)))


def quant_v(v: torch.Tensor, seq_q: int = 1, heads_q: Optional[int] = None,
            out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """V [B, S, Hkv, D] bf16 -> V~ byte buffer (layout in efq_attn.h)."""
    _bf16(v, "v")
    B, S, H, D = v.shape
    sh = Shape(B, seq_q, S, heads_q or H, H, D)
    n = vhat_bytes(sh)
    if out is None:
        out = _output(n, torch.uint8, v.device, stream)
    _check(lib().efq_quant_v_mxfp4(_ptr(v), ctypes.byref(sh), _ptr(out), out.numel(),
                                   _stream(stream)))
    return out


def attn_fwd_vhat(q, k, vhat, scale: Optional[float] = None, causal: bool = False, kind="efq",
                  params=None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    _bf16(q, "q")
    _bf16(k, "k")
    sh = shape_of(q, k)
    kind = _kind(kind)
    if scale is None:
        scale = q.shape[-1] ** -0.5
    if out is None:
        out = _output(q.shape, torch.float32, q.device, stream)
    ws, ws_n = _split_scratch(sh, causal, kind, False, stream)
    _check(lib().efq_attn_fwd_vhat_ws(_ptr(q), _ptr(k), _ptr(vhat), vhat.numel(), float(scale),
                                      int(causal), kind, _params(kind, params), _ptr(out),
                                      ctypes.byref(sh), _ptr(ws), ws_n, _stream(stream)))
    return out


def attn_fwd(q, k, v, scale: Optional[float] = None, causal: bool = False, kind="efq",
             params=None, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
             stream=None) -> torch.Tensor:
    """O = attention(q, k, v) with the chosen probability stage (fp32 out)."""
    _bf16(q, "q")
    _bf16(k, "k")
    _bf16(v, "v")
    sh = shape_of(q, k)
    kind = _kind(kind)
    if scale is None:
        scale = q.shape[-1] ** -0.5
    if out is None:
        out = _output(q.shape, torch.float32, q.device, stream)
    ws, ws_n = _workspace(sh, causal, kind, False, workspace, stream)
    _check(lib().efq_attn_fwd_ex(_ptr(q), _ptr(k), _ptr(v), float(scale), int(causal), kind,
                                 _params(kind, params), _ptr(out), ctypes.byref(sh), _ptr(ws), ws_n,
                                 _stream(stream)))
    return out


def attn_fwd_noalloc(q, k, v, out: torch.Tensor, scale: Optional[float] = None,
                     causal: bool = False, kind="efq", params=None, stream=None) -> torch.Tensor:
    """attn_fwd through the entry point that allocates nothing (V~ in the
    library's scratch array); out is the caller's fp32 BSHD tensor."""
    _bf16(q, "q")
    _bf16(k, "k")
    _bf16(v, "v")
    sh = shape_of(q, k)
    kind = _kind(kind)
    if scale is None:
        scale = q.shape[-1] ** -0.5
    _check(lib().efq_attn_fwd_noalloc(_ptr(q), _ptr(k), _ptr(v), float(scale), int(causal), kind,
                                      _params(kind, params), _ptr(out), ctypes.byref(sh),
                                      _stream(stream)))
    return out


def efq_attn_fwd(q, k, v, scale=None, causal=False, out=None, stream=None):
    """The method's entry point: EFQ-Softmax, Mean operating point."""
    sh = shape_of(q, k)
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    out = _output(q.shape, torch.float32, q.device, stream) if out is None else out
    ws, ws_n = _workspace(sh, causal, PGEN_EFQ, False, None, stream)
    _check(lib().efq_attn_fwd_ex(_ptr(q), _ptr(k), _ptr(v), float(scale), int(causal), PGEN_EFQ,
                                 Params(*PARAMS_MEAN), _ptr(out), ctypes.byref(sh), _ptr(ws), ws_n,
                                 _stream(stream)))
    return out


def efq_attn_fwd_expq(q, k, v, scale=None, causal=False, out=None, stream=None):
    """The exp-then-quantize MXFP4 baseline."""
    sh = shape_of(q, k)
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    out = _output(q.shape, torch.float32, q.device, stream) if out is None else out
    ws, ws_n = _workspace(sh, causal, PGEN_EXPQ, False, None, stream)
    _check(lib().efq_attn_fwd_ex(_ptr(q), _ptr(k), _ptr(v), float(scale), int(causal), PGEN_EXPQ,
                                 Params(*PARAMS_MEAN), _ptr(out), ctypes.byref(sh), _ptr(ws), ws_n,
                                 _stream(stream)))
    return out


def attn_fwd_dump(q, k, vhat, scale=None, causal=False, kind="efq", params=None, stream=None):
    """Attention plus the probability-stage record (codes unpacked per key)."""
    sh = shape_of(q, k)
    kind = _kind(kind)
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    B, Sq, Hq, D = q.shape
    Sk = k.shape[1]
    nblk = (Sk + 31) // 32
    dev = q.device
    out = _output(q.shape, torch.float32, dev, stream)
    codes = _output((B, Hq, Sq, nblk * 16), torch.uint8, dev, stream)
    e8 = _output((B, Hq, Sq, nblk), torch.uint8, dev, stream)
    row_m = _output((B, Hq, Sq), torch.float32, dev, stream)
    row_l = _output((B, Hq, Sq), torch.float32, dev, stream)
    _check(lib().efq_attn_fwd_dump(_ptr(q), _ptr(k), _ptr(vhat), vhat.numel(), float(scale),
                                   int(causal), kind, _params(kind, params), _ptr(out),
                                   ctypes.byref(sh), _ptr(codes), _ptr(e8), _ptr(row_m),
                                   _ptr(row_l), _stream(stream)))
    return out, codes, e8, row_m, row_l



def quant_qk(q, k, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Q, K (bf16 BSHD) -> the MXFP8 byte buffers Q^ and K^ (layout in efq_attn.h)."""
    _bf16(q, "q")
    _bf16(k, "k")
    sh = shape_of(q, k)
    qh = _output(int(lib().efq_qhat_bytes(ctypes.byref(sh))), torch.uint8, q.device, stream)
    kh = _output(int(lib().efq_khat_bytes(ctypes.byref(sh))), torch.uint8, q.device, stream)
    _check(lib().efq_quant_qk_mxfp8(_ptr(q), _ptr(k), ctypes.byref(sh), _ptr(qh), qh.numel(),
                                    _ptr(kh), kh.numel(), _stream(stream)))
    return qh, kh


def attn_fwd_qk8(qhat, khat, vhat, shape: Shape, scale: Optional[float] = None,
                 causal: bool = False, kind="efq", params=None, out: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
    """Attention on pre-quantised Q^, K^ (quant_qk) and V~ (quant_v); fp32 BSHD out."""
    kind = _kind(kind)
    if scale is None:
        scale = shape.head_dim ** -0.5
    if out is None:
        out = _output((shape.batch, shape.seq_q, shape.heads_q, shape.head_dim), torch.float32, qhat.device, stream)
    ws, ws_n = _split_scratch(shape, causal, kind, True, stream)
    _check(lib().efq_attn_fwd_qk8_ws(_ptr(qhat), qhat.numel(), _ptr(khat), khat.numel(), _ptr(vhat),
                                     vhat.numel(), float(scale), int(causal), kind,
                                     _params(kind, params), _ptr(out), ctypes.byref(shape), _ptr(ws),
                                     ws_n, _stream(stream)))
    return out


def attn_fwd_qk8_dump(qhat, khat, vhat, shape: Shape, scale=None, causal=False, kind="efq",
                      params=None, stream=None):
    """attn_fwd_qk8 plus the probability-stage record, as attn_fwd_dump."""
    kind = _kind(kind)
    scale = shape.head_dim ** -0.5 if scale is None else scale
    B, Sq, Hq, D, Sk = shape.batch, shape.seq_q, shape.heads_q, shape.head_dim, shape.seq_k
    nblk = (Sk + 31) // 32
    dev = qhat.device
    out = _output((B, Sq, Hq, D), torch.float32, dev, stream)
    codes = _output((B, Hq, Sq, nblk * 16), torch.uint8, dev, stream)
    e8 = _output((B, Hq, Sq, nblk), torch.uint8, dev, stream)
    row_m = _output((B, Hq, Sq), torch.float32, dev, stream)
    row_l = _output((B, Hq, Sq), torch.float32, dev, stream)
    _check(lib().efq_attn_fwd_qk8_dump(_ptr(qhat), qhat.numel(), _ptr(khat), khat.numel(),
                                       _ptr(vhat), vhat.numel(), float(scale), int(causal), kind,
                                       _params(kind, params), _ptr(out), ctypes.byref(shape),
                                       _ptr(codes), _ptr(e8), _ptr(row_m), _ptr(row_l),
                                       _stream(stream)))
    return out, codes, e8, row_m, row_l


def attn_fwd_lowbit(q, k, v, scale: Optional[float] = None, causal: bool = False, kind="efq",
                    params=None, out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Low-bit attention: MXFP8 Q K^T, the chosen probability stage, MXFP4 P~V.
    workspace: None, or a 256-byte aligned uint8 tensor of at least
    lowbit_workspace_bytes(shape) bytes."""
    _bf16(q, "q")
    _bf16(k, "k")
    _bf16(v, "v")
    sh = shape_of(q, k)
    kind = _kind(kind)
    if scale is None:
        scale = q.shape[-1] ** -0.5
    if out is None:
        out = _output(q.shape, torch.float32, q.device, stream)
    ws, ws_n = _workspace(sh, causal, kind, True, workspace, stream)
    _check(lib().efq_attn_fwd_lowbit_ex(_ptr(q), _ptr(k), _ptr(v), float(scale), int(causal), kind,
                                        _params(kind, params), _ptr(out), ctypes.byref(sh), _ptr(ws),
                                        ws_n, _stream(stream)))
    return out


def lowbit_workspace_bytes(shape: Shape) -> int:
    return int(lib().efq_attn_lowbit_workspace_bytes(ctypes.byref(shape)))


def qk8_natural(buf: torch.Tensor, batch: int, heads: int, seq: int, head_dim: int, scale_off: int):
    """A Q^ or K^ buffer -> (codes [B, H, seq, D], e8m0 [B, H, seq, D/32]) without padding rows."""
    sp = 64 * ((seq + 63) // 64)
    n = batch * heads * sp
    codes = buf[: n * head_dim].view(batch, heads, sp, head_dim)[:, :, :seq]
    e8 = buf[scale_off: scale_off + n * (head_dim // 32)].view(batch, heads, sp, head_dim // 32)
    return codes, e8[:, :, :seq]


def calibrate(q, k, v, o_ref, taus, hs, scale: Optional[float] = None, causal: bool = False,
              stream=None):
    """Algorithm 3 on the GPU: returns ((tau*, h*), rho [len(taus), len(hs)]).

    q, k, v: bf16 BSHD device tensors (calibration inputs); o_ref: fp32
    reference output of the shape of q.  Waits for the stream."""
    import numpy as np
    _bf16(q, "q")
    _bf16(k, "k")
    _bf16(v, "v")
    if o_ref.dtype != torch.float32 or o_ref.shape != q.shape or not o_ref.is_contiguous():
        raise ValueError("o_ref must be a contiguous fp32 tensor of the shape of q")
    sh = shape_of(q, k)
    if scale is None:
        scale = q.shape[-1] ** -0.5
    ta = np.ascontiguousarray(taus, dtype=np.float32)
    ha = np.ascontiguousarray(hs, dtype=np.float32)
    rho = np.zeros((len(ta), len(ha)), np.float64)
    best = Params(0.0, 0.0)
    nbytes = lib().efq_calibrate_workspace_bytes(ctypes.byref(sh), len(ta) * len(ha))
    ws = _output(nbytes + 256, torch.uint8, q.device, stream)
    off = (-ws.data_ptr()) % 256
    _check(lib().efq_calibrate(_ptr(q), _ptr(k), _ptr(v), float(scale), int(causal), _ptr(o_ref),
                               ctypes.byref(sh), ta.ctypes.data_as(ctypes.c_void_p), len(ta),
                               ha.ctypes.data_as(ctypes.c_void_p), len(ha),
                               rho.ctypes.data_as(ctypes.c_void_p), ctypes.byref(best),
                               ctypes.c_void_p(ws.data_ptr() + off), nbytes, _stream(stream)))
    return (best.tau, best.h), rho


# ---------------------------------------------------------------- positions, paged cache
BF16, F32 = 0, 1
_DTYPES = {torch.bfloat16: BF16, torch.float32: F32}
CACHE_BF16, CACHE_MXFP8 = 0, 1


def _place(name: str, at: int, dev: int):
    raise ValueError(f"{name} is on {'the CPU' if at < 0 else f'cuda:{at}'}, the call runs on cuda:{dev}")


def _rows(t: torch.Tensor, name: str, dtype, dev: int, heads=None, head_dim=None, tokens=None) -> Rows:
    """A [tokens, heads, head_dim] tensor with any token and head strides on device `dev`."""
    shape = t.shape
    if t.dtype is not dtype or len(shape) != 3:
        raise ValueError(f"{name} must be a {str(dtype)[6:]} tensor [tokens, heads, head_dim]")
    T, H, D = shape
    if (heads is not None and H != heads) or (head_dim is not None and D != head_dim) or (tokens is not None and T != tokens):
        raise ValueError(f"{name} has shape {tuple(shape)}, expected {(tokens, heads, head_dim)}")
    if t.get_device() != dev:
        _place(name, t.get_device(), dev)
    st, sh, sd = t.stride()
    if sd != 1 and D > 1:
        raise ValueError(f"{name} must be dense in its last dimension")
    return Rows(t.data_ptr(), st if T > 1 else 0, sh if H > 1 else 0)


def _ints(t: torch.Tensor, name: str, shape: tuple, dev: int) -> int:
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor {tuple(shape)}")
    if t.get_device() != dev:
        _place(name, t.get_device(), dev)
    return t.data_ptr()


def _rotary(pos, inv_freq, axis, interleaved, tokens: int, dev: int) -> Rotary:
    if pos.dim() not in (1, 2):
        raise ValueError("pos must be [tokens] or [axes, tokens]")
    axes = 1 if pos.dim() == 1 else pos.shape[0]
    if inv_freq.dtype is not torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
        raise ValueError("inv_freq must be a contiguous 1-D fp32 tensor")
    if inv_freq.get_device() != dev:
        _place("inv_freq", inv_freq.get_device(), dev)
    if axis is None and axes != 1:
        raise ValueError("several axes of positions need axis, the axis of every frequency")
    at = _ints(pos, "pos", (tokens,) if pos.dim() == 1 else (axes, tokens), dev)
    ax = None if axis is None else _ints(axis, "axis", inv_freq.shape, dev)
    return Rotary(inv_freq.shape[0], axes, interleaved, inv_freq.data_ptr(), ax, at)


def _tokens(t: torch.Tensor) -> torch.Tensor:
    """[B, S, H, D] as [B * S, H, D], without a copy."""
    if t.dim() != 4:
        return t
    B, S = t.shape[:2]
    if B > 1 and S > 1 and t.stride(0) != S * t.stride(1):
        raise ValueError("the batch and sequence dimensions do not merge without a copy")
    return t.as_strided((B * S, *t.shape[2:]), (t.stride(1) if S > 1 else t.stride(0), *t.stride()[2:]))


def rope(x: torch.Tensor, pos: torch.Tensor, inv_freq: torch.Tensor, axis: Optional[torch.Tensor] = None,
         interleaved: bool = False, out: Optional[torch.Tensor] = None, stream=None, _inverse: int = 0):
    """Rotary positions: x (bf16 or fp32, [tokens, heads, head_dim] or [batch,
    sequence, heads, head_dim], any token and head strides) with pair i of every
    head turned by pos[axis[i], token] * inv_freq[i].

    pos: int32 [axes, tokens] (or [tokens]); inv_freq: fp32 [pairs]; axis: int32
    [pairs], None with one axis.  interleaved: pairs of neighbours instead of
    halves.  Values behind 2 * pairs pass.  out may be x.

    Differentiable in x (any number of times): the gradient is the turn back, run
    on the stream that is current in the backward pass.  With out no gradient can
    be recorded, and the frequencies have none."""
    dtype = x.dtype
    if dtype not in _DTYPES:
        raise ValueError("x must be bf16 or fp32")
    if not x.is_cuda:
        raise ValueError("x must be a CUDA tensor")
    if (x.requires_grad or inv_freq.requires_grad) and torch.is_grad_enabled():
        if inv_freq.requires_grad:
            raise ValueError("inv_freq requires a gradient, which rope does not have")
        if out is not None:
            raise ValueError("out cannot be given where x requires a gradient")
        return _Turn.apply(x, pos, inv_freq, axis, interleaved, stream, _inverse)
    if out is None:
        out = _output(x.shape, dtype, x.device, stream)
    else:
        if out.shape != x.shape:
            raise ValueError("out must have the shape of x")
        if not out.is_inference():
            torch.autograd.graph.increment_version(out)     # what recorded out's old values must not use the new ones
    dev = torch.cuda.current_device()
    xs = _tokens(x)
    xr, yr = _rows(xs, "x", dtype, dev), _rows(_tokens(out), "out", dtype, dev)
    T, H, D = xs.shape
    rot = _rotary(pos, inv_freq, axis, interleaved, T, dev)
    _check(lib().efq_rope(xr, yr, T, H, D, _DTYPES[dtype], rot, _inverse, _stream(stream)))
    return out


class _Turn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, inv_freq, axis, interleaved, stream, inverse):
        ctx.save_for_backward(pos, inv_freq, axis)
        ctx.turn = interleaved, 1 - inverse
        return rope(x, pos, inv_freq, axis, interleaved, None, stream, inverse)

    @staticmethod
    def backward(ctx, grad):
        interleaved, inverse = ctx.turn
        grad = grad.contiguous()            # a gradient may be a broadcast one, or not aligned as rows are
        if grad.data_ptr() % 16:
            grad = grad.clone()
        back = rope(grad, *ctx.saved_tensors, interleaved, _inverse=inverse)
        return back, None, None, None, None, None, None


def rope_bwd(grad, pos, inv_freq, axis=None, interleaved=False, out=None, stream=None):
    """The gradient of rope's x from that of its output: turned back."""
    return rope(grad, pos, inv_freq, axis, interleaved, out, stream, _inverse=1)


class PagedCache:
    """Key and value pages [pages, heads_kv, page_size, head_dim]: bf16, or
    MXFP8 as uint8 codes with uint8 scales [..., head_dim / 32]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        low = k_scale is not None
        if (v_scale is not None) != low:
            raise ValueError("k_scale and v_scale come together")
        dtype = torch.uint8 if low else torch.bfloat16
        if k.dim() != 4 or v.shape != k.shape:
            raise ValueError("k and v must be [pages, heads_kv, page_size, head_dim]")
        scale_shape = (*k.shape[:3], k.shape[3] // 32)
        for t, name, d, shape in ((k, "k", dtype, k.shape), (v, "v", dtype, k.shape), (k_scale, "k_scale", dtype, scale_shape),
                                  (v_scale, "v_scale", dtype, scale_shape)):
            if t is not None and (t.dtype != d or not t.is_cuda or t.device != k.device or not t.is_contiguous() or
                                  tuple(t.shape) != tuple(shape)):
                raise ValueError(f"{name} must be a contiguous {str(d)[6:]} CUDA tensor {tuple(shape)} on {k.device}")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.heads_kv, self.page_size, self.head_dim = k.shape
        self.dev = k.get_device()
        self.c = Cache(self.pages, self.page_size, self.heads_kv, self.head_dim, CACHE_MXFP8 if low else CACHE_BF16,
                       k.data_ptr(), v.data_ptr(), k_scale.data_ptr() if low else None,
                       v_scale.data_ptr() if low else None)

    @classmethod
    def empty(cls, pages: int, page_size: int, heads_kv: int, head_dim: int, fmt: str = "bf16", device="cuda"):
        """Pages that hold nothing yet; fmt: "bf16" or "mxfp8"."""
        if fmt not in ("bf16", "mxfp8"):
            raise ValueError(f"unknown cache format {fmt!r}")
        shape = (pages, heads_kv, page_size, head_dim)
        if fmt == "bf16":
            return cls(*(torch.empty(shape, dtype=torch.bfloat16, device=device) for _ in range(2)))
        return cls(*(torch.empty(s, dtype=torch.uint8, device=device)
                     for s in (shape, shape, (*shape[:3], head_dim // 32), (*shape[:3], head_dim // 32))))


class PagedBatch:
    """The tokens of one step, for every layer of it: sequence i has seq_k[i]
    keys, the newest being the tokens q_start[i] .. q_start[i + 1] - 1, in the
    pages page_table[i] (int32 tensors on the GPU, read by the kernels).
    max_q, max_k: the most new tokens and keys of a sequence, where the host
    knows them; they choose how the work is split."""

    def __init__(self, q_start: torch.Tensor, seq_k: torch.Tensor, page_table: torch.Tensor, max_q: Optional[int] = None,
                 max_k: Optional[int] = None):
        if seq_k.dim() != 1 or not seq_k.is_cuda or page_table.dim() != 2:
            raise ValueError("seq_k must be a [sequences] CUDA tensor, page_table [sequences, width]")
        n, width = page_table.shape
        dev = seq_k.get_device()
        self.q_start, self.seq_k, self.page_table, self.dev = q_start, seq_k, page_table, dev
        self._fields = (width, int(max_q or 0), int(max_k or 0), _ints(q_start, "q_start", (n + 1,), dev),
                        _ints(seq_k, "seq_k", (n,), dev), _ints(page_table, "page_table", (n, width), dev))
        self.seqs = n
        self._last = (-1, None)

    def of(self, tokens: int) -> Batch:
        """The batch as the C entry points take it, with the calls' number of tokens."""
        last = self._last
        if last[0] != tokens:
            self._last = last = (tokens, Batch(self.seqs, tokens, *self._fields))
        return last[1]


def _together(cache: PagedCache, batch: PagedBatch) -> int:
    """The device of both, which has to be the one the call runs on."""
    dev = torch.cuda.current_device()
    if cache.dev != dev:
        _place("the cache", cache.dev, dev)
    if batch.dev != dev:
        _place("the batch", batch.dev, dev)
    return dev


def kv_append(k: torch.Tensor, v: torch.Tensor, cache: PagedCache, batch: PagedBatch, q: Optional[torch.Tensor] = None,
              q_out: Optional[torch.Tensor] = None, pos: Optional[torch.Tensor] = None,
              inv_freq: Optional[torch.Tensor] = None, axis: Optional[torch.Tensor] = None, interleaved: bool = False,
              stream=None) -> Optional[torch.Tensor]:
    """New keys and values (bf16 [tokens, heads_kv, head_dim], any strides) into
    the cache's pages (no gradient passes a cache), the keys with their positions applied when pos and
    inv_freq are given (as in rope).  With q its rows are turned too, into q_out
    (new when None; may be q), which is returned."""
    dev = _together(cache, batch)
    bf16, H, D = torch.bfloat16, cache.heads_kv, cache.head_dim
    kr = _rows(k, "k", bf16, dev, H, D)
    T = k.shape[0]
    vr = _rows(v, "v", bf16, dev, H, D, T)
    if (pos is None) != (inv_freq is None):
        raise ValueError("pos and inv_freq come together")
    rot = None if pos is None else _rotary(pos, inv_freq, axis, interleaved, T, dev)
    qr = orow = None
    heads = 0
    if q is not None:
        qr = _rows(q, "q", bf16, dev, None, D, T)
        heads = q.shape[1]
        if q_out is None:
            q_out = _output(q.shape, bf16, q.device, stream)
        orow = _rows(q_out, "q_out", bf16, dev, heads, D, T)
    elif q_out is not None:
        raise ValueError("q_out without q")
    _check(lib().efq_kv_append(kr, vr, cache.c, batch.of(T), rot, qr, heads, orow, _stream(stream)))
    return q_out


def attn_paged_workspace_bytes(cache: PagedCache, batch: PagedBatch, tokens: int, heads_q: int) -> int:
    return int(lib().efq_attn_paged_workspace_bytes(cache.c, batch.of(tokens), heads_q))


def attn_paged(q: torch.Tensor, cache: PagedCache, batch: PagedBatch, scale: Optional[float] = None, causal: bool = True,
               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Softmax attention of the new tokens q (bf16 [tokens, heads_q, head_dim],
    any strides) over the pages of their sequences; a token sees the keys up to
    its own (causal) or all.  out: bf16 or fp32 of q's shape (fp32 when None; a
    bf16 one may be q);
    lse: fp32 [tokens, heads_q] receives the log-sum-exp.  Padding tokens keep
    what out and lse held.  For inference: no gradient is recorded."""
    dev = _together(cache, batch)
    qr = _rows(q, "q", torch.bfloat16, dev, None, cache.head_dim)
    T, H, D = q.shape
    if out is None:
        out = _output(q.shape, torch.float32, q.device, stream)
    dtype = _DTYPES.get(out.dtype)
    if dtype is None:
        raise ValueError("out must be bf16 or fp32")
    orow = _rows(out, "out", out.dtype, dev, H, D, T)
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (T, H) or not lse.is_contiguous() or
                            lse.get_device() != dev):
        raise ValueError("lse must be a contiguous fp32 tensor [tokens, heads_q] on q's device")
    b, l = batch.of(T), lib()
    if workspace is None:
        n = l.efq_attn_paged_workspace_bytes(cache.c, b, H)
        if n:
            try:
                workspace = _scratch(n, stream)
            except torch.OutOfMemoryError:      # without scratch the call runs unsplit
                pass
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA tensor on q's device")
    n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(l.efq_attn_paged(qr, H, cache.c, b, D ** -0.5 if scale is None else float(scale), causal, orow, dtype,
                            None if lse is None else lse.data_ptr(), None if workspace is None else workspace.data_ptr(), n,
                            _stream(stream)))
    return out


def pgen(x: torch.Tensor, kind="efq", params=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """P-gen unit on shifted scores x [rows, cols] fp32 (CUDA)."""
    if x.dtype != torch.float32 or not x.is_cuda or not x.is_contiguous() or x.dim() != 2:
        raise ValueError("x must be a contiguous 2-D fp32 CUDA tensor")
    rows, cols = x.shape
    kind = _kind(kind)
    codes = _output((rows, (cols + 1) // 2), torch.uint8, x.device, stream)
    e8 = _output((rows, (cols + 31) // 32), torch.uint8, x.device, stream)
    _check(lib().efq_pgen(_ptr(x), rows, cols, kind, _params(kind, params), _ptr(codes), _ptr(e8),
                          _stream(stream)))
    return codes, e8


def pgen_bench(kind="efq", params=None, waves: int = 4096, iters: int = 256,
               checksum: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    kind = _kind(kind)
    if checksum is None:
        checksum = _output(waves, torch.int32, "cuda", stream)
    _check(lib().efq_pgen_bench(kind, _params(kind, params), int(waves), int(iters),
                                _ptr(checksum), _stream(stream)))
    return checksum


def clock_probe(blocks: int = 256, iters: int = 4000, out: Optional[torch.Tensor] = None,
                stream=None) -> torch.Tensor:
    """[blocks, 2] int64 on the GPU: per workgroup the s_memtime ticks (shader
    clock) and the s_memrealtime ticks (100 MHz) of an MFMA stream (the
    clock in GHz is 0.1 * col0 / col1); asynchronous on `stream`."""
    if out is None:
        out = _output((blocks, 2), torch.int64, "cuda", stream)
    if out.dtype != torch.int64 or not out.is_cuda or out.numel() < 2 * blocks or not out.is_contiguous():
        raise ValueError("out must be a contiguous int64 CUDA tensor of at least 2 * blocks elements")
    _check(lib().efq_clock_probe(int(blocks), int(iters), _ptr(out), _stream(stream)))
    return out


def unpack_nibbles(packed: torch.Tensor) -> torch.Tensor:
    """[..., n] bytes -> [..., 2n] codes (low nibble first)."""
    p = packed.to(torch.int16)
    return torch.stack([p & 0xF, p >> 4], dim=-1).flatten(-2).to(torch.uint8)


def vhat_natural(vhat: torch.Tensor, shape: Shape):
    """Reorder a V~ buffer to (codes [B, Hkv, nb*32, D] one per byte, e8m0
    [B, Hkv, nb, D]) in key order (layout stated in efq_attn.h)."""
    B, H, D = shape.batch, shape.heads_kv, shape.head_dim
    nb = 2 * ((shape.seq_k + 63) // 64)
    off = vhat_scale_offset(shape)
    codes = vhat[: B * H * nb * D * 16].view(B, H, nb, D, 16)
    nib = unpack_nibbles(codes)                        # [B, H, nb, D, 32] nibble order
    t = torch.arange(32)
    e = (8 * (2 * ((t >> 2) & 1) + (t >> 4)) + 2 * (t & 3) + ((t >> 3) & 1)).to(vhat.device)
    keyed = nib[..., e]                                # [..., 32] key order
    codes_nat = keyed.permute(0, 1, 2, 4, 3).reshape(B, H, nb * 32, D)
    # scale plane: byte (d % 32) * (D / 32) + d / 32 of each block
    e8 = vhat[off: off + B * H * nb * D].view(B, H, nb, 32, D // 32)
    e8 = e8.permute(0, 1, 2, 4, 3).reshape(B, H, nb, D)
    return codes_nat, e8

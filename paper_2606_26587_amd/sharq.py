"""Python binding of libsharq.so (the HIP kernels behind include/sharq.h).

Argument marshalling only: buffers are torch tensors on the GPU (torch is used
for device memory and streams), every computation runs in the library's
kernels.  A call runs on `stream` (a torch.cuda.Stream; None: the current one),
and the buffers that it is not given are allocated there: like any tensor of
that stream, they are marked with record_stream before they are dropped while
another stream still uses them.  Importing this module raises if the library has not been built;
there is no fallback path.
"""

from __future__ import annotations

import contextlib
import ctypes
import functools
import operator
import os
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libsharq.so")

OK, EINVAL, EUNSUPPORTED, EALIGN, EHIP = 0, 1, 2, 3, 4
MXFP4, NVFP4, HIF4 = 0, 1, 2
BF16, F16, F32 = 0, 1, 2

_FMT = {"mx": MXFP4, "mxfp4": MXFP4, "nv": NVFP4, "nvfp4": NVFP4, "hif4": HIF4}
#: path combinations (sharq_mode): the method, and the ablation modes
MODES = {"sharq": 0, "sparse": 1, "dense": 2, "dense_dense": 3, "sparse_sparse": 4}
_DT = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}
#: E8M0 scale rules of MXFP4 (sharq_scale_rule)
SCALE_RULES = {"floor": 0, "ceil": 1}


class SharqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib.sharq_status_str(status).decode()} (status {status})")


class Pattern(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("m", ctypes.c_int32), ("pairs", ctypes.c_int32)]


class ActStruct(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("K", ctypes.c_int64), ("fmt", ctypes.c_int), ("nm", Pattern),
                ("sp_codes", ctypes.c_void_p), ("sp_meta", ctypes.c_void_p), ("sp_scale", ctypes.c_void_p),
                ("dn_codes", ctypes.c_void_p), ("dn_scale", ctypes.c_void_p), ("tensor_scale", ctypes.c_void_p),
                ("mode", ctypes.c_int), ("dn_meta", ctypes.c_void_p), ("sp_dense", ctypes.c_void_p),
                ("scale_rule", ctypes.c_int), ("dbg_mask", ctypes.c_void_p), ("dbg_r", ctypes.c_void_p)]


class WeightStruct(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("K", ctypes.c_int64), ("experts", ctypes.c_int64), ("fmt", ctypes.c_int),
                ("codes", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("scale_dn", ctypes.c_void_p),
                ("tensor_scale", ctypes.c_void_p), ("scale_rule", ctypes.c_int)]


class KVCacheStruct(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("fmt", ctypes.c_int), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("scale_rule", ctypes.c_int)]


class KVBatchStruct(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_int64), ("rows", ctypes.c_int64), ("max_rows", ctypes.c_int64),
                ("max_len", ctypes.c_int64), ("ld_table", ctypes.c_int64), ("row_offsets", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("page_table", ctypes.c_void_p)]


class AttnStruct(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("window", ctypes.c_int64), ("sinks", ctypes.c_int64),
                ("prefix_table", ctypes.c_void_p), ("prefix_len", ctypes.c_int64)]


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is not built; run `python -m paper_2606_26587_amd.build`")
    L = ctypes.CDLL(_LIB_PATH)
    c_i64, c_vp, c_f = ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
    L.sharq_version.restype = ctypes.c_char_p
    L.sharq_version.argtypes = []
    L.sharq_status_str.restype = ctypes.c_char_p
    L.sharq_status_str.argtypes = [ctypes.c_int]
    L.sharq_act_buffer_bytes.restype = ctypes.c_size_t
    L.sharq_act_buffer_bytes.argtypes = [c_i64, c_i64, ctypes.c_int, Pattern, ctypes.c_int32]
    L.sharq_act_buffer_bytes_mode.restype = ctypes.c_size_t
    L.sharq_act_buffer_bytes_mode.argtypes = [c_i64, c_i64, ctypes.c_int, Pattern, ctypes.c_int, ctypes.c_int32]
    L.sharq_weight_buffer_bytes.restype = ctypes.c_size_t
    L.sharq_weight_buffer_bytes.argtypes = [c_i64, c_i64, ctypes.c_int, ctypes.c_int32]
    L.sharq_quantize_weight.restype = ctypes.c_int
    L.sharq_quantize_weight.argtypes = [c_vp, ctypes.c_int, c_i64, c_i64, c_i64, ctypes.POINTER(WeightStruct), c_vp]
    L.sharq_prepare.restype = ctypes.c_int
    L.sharq_prepare.argtypes = [c_vp, ctypes.c_int, c_i64, c_i64, c_i64, c_vp, c_f, Pattern, ctypes.c_int, c_vp,
                                ctypes.POINTER(ActStruct), c_vp]
    L.sharq_prepare_residual.restype = ctypes.c_int
    L.sharq_prepare_residual.argtypes = [c_vp, c_vp, c_vp, ctypes.c_int, c_i64, c_i64, c_i64, c_i64, c_i64, c_vp, c_f,
                                         Pattern, ctypes.c_int, c_vp, ctypes.POINTER(ActStruct), c_vp]
    L.sharq_prepare_silu_mul.restype = ctypes.c_int
    L.sharq_prepare_silu_mul.argtypes = [c_vp, c_vp, c_vp, ctypes.c_int, c_i64, c_i64, c_i64, c_i64, c_i64, Pattern,
                                         ctypes.c_int, c_vp, ctypes.POINTER(ActStruct), c_vp]
    L.sharq_linear.restype = ctypes.c_int
    L.sharq_linear.argtypes = [ctypes.POINTER(ActStruct), ctypes.POINTER(WeightStruct), c_vp, ctypes.c_int, c_i64,
                               c_vp]
    L.sharq_prepare_linear.restype = ctypes.c_int
    L.sharq_prepare_linear.argtypes = [c_vp, ctypes.c_int, c_i64, c_i64, c_i64, c_vp, c_f, Pattern, ctypes.c_int, c_vp,
                                       ctypes.POINTER(ActStruct), ctypes.POINTER(WeightStruct), c_vp, ctypes.c_int,
                                       c_i64, c_vp]
    L.sharq_linear_grouped.restype = ctypes.c_int
    L.sharq_linear_grouped.argtypes = [ctypes.POINTER(ActStruct), c_vp, c_vp, c_i64, ctypes.POINTER(WeightStruct),
                                       c_vp, ctypes.c_int, c_i64, c_vp]
    cache_p, batch_p, attn_p = (ctypes.POINTER(t) for t in (KVCacheStruct, KVBatchStruct, AttnStruct))
    L.sharq_kv_buffer_bytes.restype = ctypes.c_size_t
    L.sharq_kv_buffer_bytes.argtypes = [cache_p, ctypes.c_int32]
    L.sharq_kv_append.restype = ctypes.c_int
    L.sharq_kv_append.argtypes = [c_vp, c_vp, c_vp, ctypes.c_int, c_i64, c_i64, c_i64, c_i64, c_vp, c_vp, c_i64, c_vp,
                                  cache_p, batch_p, c_vp, c_i64, c_vp]
    L.sharq_kv_read.restype = ctypes.c_int
    L.sharq_kv_read.argtypes = [cache_p, batch_p, c_vp, c_i64, c_vp, c_i64, ctypes.c_int, c_vp]
    L.sharq_attention_workspace_bytes.restype = ctypes.c_size_t
    L.sharq_attention_workspace_bytes.argtypes = [cache_p, batch_p, attn_p, c_i64]
    L.sharq_attention.restype = ctypes.c_int
    L.sharq_attention.argtypes = [c_vp, ctypes.c_int, c_i64, c_i64, cache_p, batch_p, attn_p, c_vp, c_i64, c_vp, c_vp,
                                  ctypes.c_size_t, c_vp]
    return L


lib = _load()


def _check(status: int, where: str):
    if status != OK:
        raise SharqError(status, where)


# The calls below run once per layer and decode step, where a kernel takes 5 to
# 10 us: they pass plain integers (ctypes converts them by argtypes) and ask
# torch for the current stream's handle without building a Stream object (2.9
# us of the 9.0 us a sharq_linear call took on the host; 6.0 us after).

def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream_handle(c=torch._C):
    """The function that gives the current stream's handle: torch's raw accessors, which are not part of its
    public interface, or the Stream object where a torch has none."""
    raw, device = getattr(c, "_cuda_getCurrentRawStream", None), getattr(c, "_cuda_getDevice", None)
    if raw is None or device is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(device())


_current = _stream_handle()


def _stream(stream):
    return _current() if stream is None else stream.cuda_stream


_CURRENT = contextlib.nullcontext()


def _on(stream):
    """The context in which a call allocates its buffers: its own stream, whose work in the order of the calls is what
    the allocator relies on when it hands a block out again.  (From another stream's blocks one could come whose last
    reader there is still to run.)"""
    return _CURRENT if stream is None else torch.cuda.stream(stream)


# ---------------------------------------------------------------------------
# Containers
# ---------------------------------------------------------------------------

@dataclass
class PreparedAct:
    """Output of sharq_prepare: the compressed backbone and the residual (device
    buffers).  In the ablation modes path 1 lives in the sp_* buffers and path 2
    in the dn_* buffers (dn_meta: a sparse path 2)."""
    rows: int
    K: int
    fmt: int
    n: int
    m: int
    sp_codes: torch.Tensor
    sp_meta: torch.Tensor
    sp_scale: torch.Tensor
    dn_codes: torch.Tensor
    dn_scale: torch.Tensor
    tensor_scale: Optional[torch.Tensor] = None
    pairs: bool = False
    mode: int = 0
    dn_meta: Optional[torch.Tensor] = None
    sp_dense: Optional[torch.Tensor] = None   # MXFP4/NVFP4: the backbone's dense copy for the main GEMM
    scale_rule: int = 0                       # MXFP4: E8M0 rule (SCALE_RULES)
    dbg_mask: Optional[torch.Tensor] = None   # debug: keep bits, 4 bytes per 32 positions
    dbg_r: Optional[torch.Tensor] = None      # debug: RMSNorm r per row (fp32)

    def struct(self) -> ActStruct:
        return ActStruct(self.rows, self.K, self.fmt, Pattern(self.n, self.m, int(self.pairs)), _ptr(self.sp_codes),
                         _ptr(self.sp_meta), _ptr(self.sp_scale), _ptr(self.dn_codes), _ptr(self.dn_scale),
                         _ptr(self.tensor_scale), self.mode, _ptr(self.dn_meta), _ptr(self.sp_dense), self.scale_rule,
                         _ptr(self.dbg_mask), _ptr(self.dbg_r))


@dataclass
class QuantWeight:
    """Shared FP4 weight payload with its path-specific scale views (device buffers)."""
    N: int
    K: int
    experts: int
    fmt: int
    codes: torch.Tensor
    scale: torch.Tensor
    scale_dn: torch.Tensor
    tensor_scale: Optional[torch.Tensor] = None
    scale_rule: int = 0                       # MXFP4: E8M0 rule used by sharq_quantize_weight

    def struct(self) -> WeightStruct:
        return WeightStruct(self.N, self.K, self.experts, self.fmt, self.codes.data_ptr(), self.scale.data_ptr(),
                            self.scale_dn.data_ptr(),
                            None if self.tensor_scale is None else self.tensor_scale.data_ptr(), self.scale_rule)


KV_FORMATS = {"bf16": 0, "mx": 1, "mxfp4": 1}


# The two descriptors below are used by every layer of a decode step: they are
# checked and turned into their C structures once, and cannot be changed after
# (the tensors' contents can).

@dataclass(frozen=True)
class KVCache:
    """A paged key/value cache (device buffers; sharq_kv_cache in include/sharq.h).
    fmt "bf16": k, v [pages, kv_heads, page_size, head_dim]; "mx": k, v uint8
    codes [..., head_dim / 2] and their E8M0 scales uint8 [..., head_dim / 32]."""
    fmt: str
    k: torch.Tensor
    v: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None
    scale_rule: str = "floor"                 # "mx": E8M0 rule of sharq_kv_append (SCALE_RULES)

    def __post_init__(self):
        mx = KV_FORMATS[self.fmt] == 1
        shape = tuple(self.k.shape)
        ok = len(shape) == 4 and tuple(self.v.shape) == shape
        for t in (self.k, self.v):
            ok = ok and t.dtype == (torch.uint8 if mx else torch.bfloat16)
        if mx and ok:
            ok = self.k_scale is not None and self.v_scale is not None
            for t in (self.k_scale, self.v_scale):
                ok = ok and t.dtype == torch.uint8 and tuple(t.shape) == shape[:3] + (shape[3] // 16,)
        given = [t for t in (self.k, self.v, self.k_scale, self.v_scale) if t is not None]
        if not ok or any(not t.is_contiguous() or t.device != self.k.device for t in given):
            raise SharqError(EINVAL, "KVCache")
        pages, kv_heads, page_size = shape[:3]
        head_dim = shape[3] * 2 if mx else shape[3]
        struct = KVCacheStruct(pages, page_size, kv_heads, head_dim, KV_FORMATS[self.fmt], self.k.data_ptr(),
                               self.v.data_ptr(), _ptr(self.k_scale), _ptr(self.v_scale),
                               SCALE_RULES[self.scale_rule])
        self.__dict__.update(pages=pages, kv_heads=kv_heads, page_size=page_size, head_dim=head_dim,
                             width=kv_heads * head_dim, device_index=self.k.get_device(), ref=ctypes.byref(struct))


@dataclass(frozen=True)
class KVBatch:
    """The sequences of a call (sharq_kv_batch): row_offsets int32 [seqs + 1], lens
    int32 [seqs] (the call's rows among them), page_table int32 [seqs, n], on the
    GPU; the rows of the row tensors, and the host's bounds of a sequence's rows and
    length (max_len at most n pages; the attention's work is split by these bounds,
    so far above the sequences' own they cost time)."""
    row_offsets: torch.Tensor
    lens: torch.Tensor
    page_table: torch.Tensor
    rows: int
    max_rows: int
    max_len: int

    def __post_init__(self):
        seqs = self.lens.numel()
        for t, shape in ((self.row_offsets, (seqs + 1,)), (self.lens, (seqs,)), (self.page_table[:, :0], (seqs, 0))):
            if t.dtype != torch.int32 or tuple(t.shape) != shape or t.device != self.lens.device:
                raise SharqError(EINVAL, "KVBatch")
        if not (self.row_offsets.is_contiguous() and self.lens.is_contiguous() and
                (self.page_table.shape[1] <= 1 or self.page_table.stride(1) == 1) and
                (seqs <= 1 or self.page_table.stride(0) >= self.page_table.shape[1])):
            raise SharqError(EINVAL, "KVBatch")

        # the stride of a single sequence means nothing: its row is as long as the table is wide
        ld = self.page_table.stride(0) if seqs > 1 else self.page_table.shape[1]
        struct = KVBatchStruct(seqs, self.rows, self.max_rows, self.max_len, ld, self.row_offsets.data_ptr(),
                               self.lens.data_ptr(), self.page_table.data_ptr())
        # the library is told the stride alone: that the table is as wide as max_len takes is checked here, per call
        # (the page size is the cache's); where nothing is looked up, any width will do
        least = -1 if seqs == 0 or self.rows == 0 else self.max_len
        self.__dict__.update(device_index=self.lens.get_device(), table_pages=self.page_table.shape[1],
                             table_tokens=least, ref=ctypes.byref(struct))


def alloc_kv_cache(pages: int, page_size: int, kv_heads: int, head_dim: int, fmt: str = "bf16", device="cuda",
                   scale_rule: str = "floor") -> KVCache:
    """An empty paged cache; its pages are read only where something was appended."""
    shape = (pages, kv_heads, page_size)
    if KV_FORMATS[fmt] == 0:
        return KVCache(fmt, *(torch.empty(shape + (head_dim,), dtype=torch.bfloat16, device=device) for _ in "kv"),
                       scale_rule=scale_rule)
    return KVCache(fmt, *(torch.empty(shape + (head_dim // n,), dtype=torch.uint8, device=device)
                          for n in (2, 2, 32, 32)), scale_rule=scale_rule)


def alloc_act(rows: int, K: int, n: int = 2, m: int = 4, fmt="mx", device="cuda", pairs: bool = False,
              mode="sharq", dense_backbone: bool = False, dense_only: bool = False, scale_rule="floor",
              debug: bool = False) -> PreparedAct:
    """Device buffers of a prepared activation (flat, panel-major; see include/sharq.h).
    pairs=True: n:m selection in pairs (4:8 in pairs).  mode: a key of MODES
    (or its id); buffers a mode does not use are empty.  dense_backbone=True
    (MXFP4, NVFP4): also the backbone's dense copy that the main GEMM reads without
    expanding it; dense_only=True: that copy instead of the compressed
    backbone.  scale_rule: "floor" or "ceil" (MXFP4 E8M0 rule).  debug=True:
    also the keep-mask and per-row r debug outputs."""
    f = _FMT[fmt] if isinstance(fmt, str) else fmt
    md = MODES[mode] if isinstance(mode, str) else int(mode)
    sizes = [lib.sharq_act_buffer_bytes_mode(rows, K, f, Pattern(n, m, int(pairs)), md, w) for w in range(6)]
    used = sizes[:5] if md == 0 else [z for z in sizes if z]
    if K <= 0 or K % 32 or (rows > 0 and (not used or min(used) == 0)):
        raise SharqError(EINVAL, "alloc_act")
    bufs = [torch.empty(sz, dtype=torch.uint8, device=device) for sz in sizes]
    ts = torch.empty(1, dtype=torch.float32, device=device) if f == NVFP4 else None
    spd = torch.empty(rows * K // 2, dtype=torch.uint8, device=device) if (dense_backbone or dense_only) else None
    if dense_only:
        bufs[0] = bufs[1] = None
    rule = SCALE_RULES[scale_rule] if isinstance(scale_rule, str) else int(scale_rule)
    dbg_mask = torch.empty(rows * K // 8, dtype=torch.uint8, device=device) if debug else None
    dbg_r = torch.empty(rows, dtype=torch.float32, device=device) if debug else None
    return PreparedAct(rows, K, f, n, m, *bufs[:5], tensor_scale=ts, pairs=pairs, mode=md, dn_meta=bufs[5],
                       sp_dense=spd, scale_rule=rule, dbg_mask=dbg_mask, dbg_r=dbg_r)


def alloc_weight(N: int, K: int, fmt="mx", experts: int = 1, device="cuda", scale_rule="floor") -> QuantWeight:
    """Device buffers of a quantized weight, one flat panel-major row per expert."""
    f = _FMT[fmt] if isinstance(fmt, str) else fmt
    codes = torch.empty((experts, N * K // 2), dtype=torch.uint8, device=device)
    scale = torch.empty((experts, N * K // (16 if f == HIF4 else 32)), dtype=torch.uint8, device=device)
    scale_dn = scale if f != NVFP4 else torch.empty((experts, N * K // 16), dtype=torch.uint8, device=device)
    ts = torch.empty(experts, dtype=torch.float32, device=device) if f == NVFP4 else None
    rule = SCALE_RULES[scale_rule] if isinstance(scale_rule, str) else int(scale_rule)
    return QuantWeight(N, K, experts, f, codes, scale, scale_dn, ts, rule)


# ---------------------------------------------------------------------------
# Entry points (same names as the C ABI)
# ---------------------------------------------------------------------------

def sharq_quantize_weight(w: torch.Tensor, fmt="mx", out: Optional[QuantWeight] = None, stream=None,
                          scale_rule="floor") -> QuantWeight:
    """Quantize W [N, K] (bf16 or fp32, on the GPU) into the shared FP4 payload
    (scale_rule: the MXFP4 E8M0 rule, ignored when `out` is given)."""
    N, K = w.shape
    if out is None:
        with _on(stream):
            out = alloc_weight(N, K, fmt, 1, w.device, scale_rule)
    ws = out.struct()
    _check(lib.sharq_quantize_weight(_ptr(w), _DT.get(w.dtype, -1), N, K, w.stride(0), ctypes.byref(ws),
                                     _stream(stream)), "sharq_quantize_weight")
    return out


def sharq_prepare(x: torch.Tensor, gamma: Optional[torch.Tensor], eps: float = 1e-6, n: int = 2, m: int = 4,
                  fmt="mx", tensor_scale_in: Optional[torch.Tensor] = None, out: Optional[PreparedAct] = None,
                  stream=None, pairs: bool = False, mode="sharq", scale_rule="floor") -> PreparedAct:
    """Fused preparation of activation rows X [M, K] (bf16, on the GPU).
    pairs=True: n:m selection in pairs (NVFP4's 4:8 in pairs).  mode, scale_rule:
    the path combination (MODES) and the MXFP4 E8M0 rule (SCALE_RULES), both
    ignored when `out` is given, which carries them."""
    M, K = x.shape
    if out is None:
        with _on(stream):
            out = alloc_act(M, K, n, m, fmt, x.device, pairs, mode, scale_rule=scale_rule)
    f = _FMT[fmt] if isinstance(fmt, str) else fmt
    st = out.struct()
    _check(lib.sharq_prepare(_ptr(x), _DT.get(x.dtype, -1), M, K, x.stride(0), _ptr(gamma), eps,
                             Pattern(n, m, int(pairs)), f, _ptr(tensor_scale_in), ctypes.byref(st), _stream(stream)),
           "sharq_prepare")
    return out


def sharq_prepare_residual(x: torch.Tensor, residual: torch.Tensor, gamma: Optional[torch.Tensor], eps: float = 1e-6,
                           n: int = 2, m: int = 4, fmt="mx", h_out: Optional[torch.Tensor] = None,
                           tensor_scale_in: Optional[torch.Tensor] = None, out: Optional[PreparedAct] = None,
                           stream=None, pairs: bool = False):
    """Residual add fused into the preparation: h = bf16(x + residual) is
    written to h_out (a new tensor, or e.g. `residual` itself for an in-place
    update) and prepared.  Returns (prepared activation, h)."""
    M, K = x.shape
    if out is None:
        with _on(stream):
            out = alloc_act(M, K, n, m, fmt, x.device, pairs)
    if h_out is None:
        with _on(stream):
            h_out = torch.empty_like(x)
    f = _FMT[fmt] if isinstance(fmt, str) else fmt
    st = out.struct()
    _check(lib.sharq_prepare_residual(_ptr(x), _ptr(residual), _ptr(h_out), _DT.get(x.dtype, -1), M, K, x.stride(0),
                                      residual.stride(0), h_out.stride(0), _ptr(gamma), eps,
                                      Pattern(n, m, int(pairs)), f, _ptr(tensor_scale_in), ctypes.byref(st),
                                      _stream(stream)), "sharq_prepare_residual")
    return out, h_out


def sharq_prepare_silu_mul(gate: torch.Tensor, up: torch.Tensor, n: int = 2, m: int = 4, fmt="mx",
                           h_out: Optional[torch.Tensor] = None, tensor_scale_in: Optional[torch.Tensor] = None,
                           out: Optional[PreparedAct] = None, stream=None, pairs: bool = False) -> PreparedAct:
    """SiLU.mul fused into the preparation of a down projection's input:
    h = bf16(SiLU(gate) * up) is prepared (and written to h_out when given)."""
    M, K = gate.shape
    if out is None:
        with _on(stream):
            out = alloc_act(M, K, n, m, fmt, gate.device, pairs)
    f = _FMT[fmt] if isinstance(fmt, str) else fmt
    st = out.struct()
    _check(lib.sharq_prepare_silu_mul(_ptr(gate), _ptr(up), _ptr(h_out), _DT.get(gate.dtype, -1), M, K,
                                      gate.stride(0), up.stride(0), h_out.stride(0) if h_out is not None else K,
                                      Pattern(n, m, int(pairs)), f, _ptr(tensor_scale_in), ctypes.byref(st),
                                      _stream(stream)), "sharq_prepare_silu_mul")
    return out


def sharq_linear(a: PreparedAct, w: QuantWeight, out: Optional[torch.Tensor] = None, dtype=torch.bfloat16,
                 stream=None) -> torch.Tensor:
    """Y [rows, N] = backbone GEMM + residual GEMM over the shared weight."""
    if out is None:
        with _on(stream):
            out = torch.empty((a.rows, w.N), dtype=dtype, device=a.dn_codes.device)
    ast, wst = a.struct(), w.struct()
    _check(lib.sharq_linear(ctypes.byref(ast), ctypes.byref(wst), _ptr(out), _DT.get(out.dtype, -1),
                            out.stride(0) if out.dim() == 2 else w.N, _stream(stream)), "sharq_linear")
    return out


def sharq_prepare_linear(x: torch.Tensor, gamma: Optional[torch.Tensor], w: QuantWeight, eps: float = 1e-6, n: int = 2,
                         m: int = 4, fmt="mx", act: Optional[PreparedAct] = None, out: Optional[torch.Tensor] = None,
                         dtype=torch.bfloat16, tensor_scale_in: Optional[torch.Tensor] = None, stream=None,
                         pairs: bool = False, scale_rule="floor"):
    """Preparation of X [M, K] into `act` and Y = SharQ(act, w) in one call
    (one kernel for a few rows).  Returns (prepared activation, Y)."""
    M, K = x.shape
    if act is None:
        with _on(stream):
            act = alloc_act(M, K, n, m, fmt, x.device, pairs, scale_rule=scale_rule)
    if out is None:
        with _on(stream):
            out = torch.empty((M, w.N), dtype=dtype, device=x.device)
    f = _FMT[fmt] if isinstance(fmt, str) else fmt
    ast, wst = act.struct(), w.struct()
    _check(lib.sharq_prepare_linear(_ptr(x), _DT.get(x.dtype, -1), M, K, x.stride(0), _ptr(gamma), eps,
                                    Pattern(n, m, int(pairs)), f, _ptr(tensor_scale_in), ctypes.byref(ast),
                                    ctypes.byref(wst), _ptr(out), _DT.get(out.dtype, -1),
                                    out.stride(0) if out.dim() == 2 else w.N, _stream(stream)), "sharq_prepare_linear")
    return act, out


def sharq_linear_grouped(a: PreparedAct, row_index: Optional[torch.Tensor], expert_offsets: torch.Tensor, total: int,
                         w: QuantWeight, out: Optional[torch.Tensor] = None, dtype=torch.bfloat16,
                         stream=None) -> torch.Tensor:
    """Mixture-of-experts form: Y[i] = SharQ(A[row_index[i]], W_e) for i in expert e's slice."""
    if out is None:
        with _on(stream):
            out = torch.empty((total, w.N), dtype=dtype, device=a.dn_codes.device)
    ast, wst = a.struct(), w.struct()
    _check(lib.sharq_linear_grouped(ctypes.byref(ast), _ptr(row_index), _ptr(expert_offsets), total,
                                    ctypes.byref(wst), _ptr(out), _DT.get(out.dtype, -1),
                                    out.stride(0) if out.dim() == 2 else w.N, _stream(stream)),
           "sharq_linear_grouped")
    return out


_BF = torch.bfloat16


def _rows(t: torch.Tensor, rows: int, width: int, dev: int, where: str) -> int:
    """Row stride of a row tensor [rows, width], bf16 on device `dev`, its rows contiguous."""
    if t.dtype is _BF and t.shape == (rows, width) and t.get_device() == dev:
        ld, inner = t.stride()
        if inner == 1 or width <= 1:
            return ld if rows > 1 else width   # the stride of a single row means nothing
    raise SharqError(EINVAL, where)


_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _here(cache: KVCache, batch: KVBatch, where: str):
    """The kernels are launched on the current device: the buffers must be its own."""
    dev = cache.device_index
    if dev < 0 or dev != batch.device_index or dev != _device():
        raise SharqError(EINVAL, where)


def _table(cache: KVCache, batch: KVBatch, where: str):
    """Every token that the call may look up has a column in the page table.  A table that is a slice of a wider one has
    a stride above its width: behind a row's own entries come the parent's, and behind the last row's perhaps nothing."""
    if batch.table_tokens > batch.table_pages * cache.page_size:
        raise SharqError(EINVAL, where)


def sharq_kv_append(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, cache: KVCache, batch: KVBatch,
                    cos: Optional[torch.Tensor] = None, sin: Optional[torch.Tensor] = None,
                    positions: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                    stream=None) -> Optional[torch.Tensor]:
    """Rotate the rows' queries and keys (cos, sin: fp32 [positions, head_dim / 2]; None: no rotation) and put keys and
    values into the cache.  q, k, v: bf16 [rows, heads * head_dim], e.g. slices of the qkv projection's output.
    Returns the rotated queries (q_out; `q` itself for an in-place update), None without q."""
    where = "sharq_kv_append"
    _here(cache, batch, where)
    _table(cache, batch, where)
    rows, dev = batch.rows, cache.device_index
    ldk, ldv = _rows(k, rows, cache.width, dev, where), _rows(v, rows, cache.width, dev, where)
    heads = ldq = ldo = angles = 0
    if q is not None:
        width = q.shape[-1]
        heads, rest = divmod(width, cache.head_dim)
        ldq = _rows(q, rows, width, dev, where)
        if rest:
            raise SharqError(EINVAL, where)
        if q_out is None:
            with _on(stream):
                q_out = torch.empty((rows, width), dtype=q.dtype, device=q.device)
        ldo = _rows(q_out, rows, width, dev, where)
    if (cos is None) != (sin is None):
        raise SharqError(EINVAL, where)
    if cos is not None:
        angles = cos.shape[0]
        shape = (angles, cache.head_dim // 2)
        if not (cos.dtype is sin.dtype is torch.float32 and cos.shape == sin.shape == shape and cos.is_contiguous()
                and sin.is_contiguous() and cos.get_device() == sin.get_device() == dev):
            raise SharqError(EINVAL, where)
    if positions is not None and (positions.dtype is not torch.int32 or positions.shape != (rows,)
                                  or not positions.is_contiguous() or positions.get_device() != dev):
        raise SharqError(EINVAL, where)
    status = lib.sharq_kv_append(_ptr(q), k.data_ptr(), v.data_ptr(), BF16, heads, ldq, ldk, ldv, _ptr(cos), _ptr(sin),
                                 angles, _ptr(positions), cache.ref, batch.ref, None if q is None else q_out.data_ptr(),
                                 ldo, _stream(stream))
    if status:
        raise SharqError(status, where)
    return None if q is None else q_out


def sharq_kv_read(cache: KVCache, batch: KVBatch, k_out: Optional[torch.Tensor] = None,
                  v_out: Optional[torch.Tensor] = None, stream=None):
    """The rows' cached keys and values as bf16 [rows, kv_heads * head_dim] (padding rows are left as they are)."""
    where = "sharq_kv_read"
    _here(cache, batch, where)
    _table(cache, batch, where)
    shape = (batch.rows, cache.width)
    if k_out is None:
        with _on(stream):
            k_out = torch.empty(shape, dtype=_BF, device=cache.k.device)
    if v_out is None:
        with _on(stream):
            v_out = torch.empty(shape, dtype=_BF, device=cache.k.device)
    ldk, ldv = (_rows(t, *shape, cache.device_index, where) for t in (k_out, v_out))
    _check(lib.sharq_kv_read(cache.ref, batch.ref, k_out.data_ptr(), ldk, v_out.data_ptr(), ldv, BF16,
                             _stream(stream)), where)
    return k_out, v_out


@functools.lru_cache(maxsize=64)
def _attn_ref(scale: float, window: int, sinks: int):
    """A reference to the C structure of a call without a shared prefix: a layer's are always the same.  Plain numbers
    only: anything else would be kept by its identity, whatever it holds later."""
    return ctypes.byref(AttnStruct(scale, window, sinks, None, 0))


def attention_workspace_bytes(cache: KVCache, batch: KVBatch, q_heads: int, window: int = 0, sinks: int = 0,
                              prefix_len: int = 0) -> int:
    """Bytes of workspace of sharq_attention for these sizes."""
    ts = AttnStruct(1.0, window, sinks, None, prefix_len)
    return lib.sharq_attention_workspace_bytes(cache.ref, batch.ref, ctypes.byref(ts), q_heads)


def sharq_attention(q: torch.Tensor, cache: KVCache, batch: KVBatch, scale: Optional[float] = None, window: int = 0,
                    sinks: int = 0, prefix_table: Optional[torch.Tensor] = None, prefix_len: int = 0,
                    out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Causal attention of the rows over their cached sequences (their own keys and values appended before).
    scale: 1 / sqrt(head_dim) by default; window: 0, all tokens; sinks: first tokens that stay visible;
    prefix_table, prefix_len: pages that all sequences begin with, read once for all.  lse: fp32 [rows, q_heads], filled
    when given.  workspace: a buffer of attention_workspace_bytes, allocated here when needed and None."""
    where = "sharq_attention"
    _here(cache, batch, where)
    _table(cache, batch, where)
    rows, dev, width = batch.rows, cache.device_index, q.shape[-1]
    heads, rest = divmod(width, cache.head_dim)
    ldq = _rows(q, rows, width, dev, where)
    if rest:
        raise SharqError(EINVAL, where)
    if out is None:
        with _on(stream):
            out = torch.empty((rows, width), dtype=q.dtype, device=q.device)
    ldo = _rows(out, rows, width, dev, where)
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (rows, heads) or not lse.is_contiguous()
                            or lse.get_device() != dev):
        raise SharqError(EINVAL, where)
    if prefix_table is not None and (prefix_table.dtype is not torch.int32 or not prefix_table.is_contiguous()
                                     or prefix_table.numel() * cache.page_size < prefix_len
                                     or prefix_table.get_device() != dev):
        raise SharqError(EINVAL, where)
    if scale is None:
        scale = cache.head_dim ** -0.5
    if prefix_len or prefix_table is not None:
        ts = ctypes.byref(AttnStruct(scale, window, sinks, _ptr(prefix_table), prefix_len))
    else:
        ts = _attn_ref(float(scale), operator.index(window), operator.index(sinks))
    size = 0
    if workspace is None:
        size = lib.sharq_attention_workspace_bytes(cache.ref, batch.ref, ts, heads)
        if size:   # freed on return, and taken again only behind the call
            with _on(stream):
                workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise SharqError(EINVAL, where)
    else:
        size = workspace.nbytes
    status = lib.sharq_attention(q.data_ptr(), BF16, heads, ldq, cache.ref, batch.ref, ts, out.data_ptr(), ldo,
                                 _ptr(lse), _ptr(workspace), size, _stream(stream))
    if status:
        raise SharqError(status, where)
    return out


def stack_weights(ws: Sequence[QuantWeight]) -> QuantWeight:
    """Stack per-expert weights of one shape into one [experts] payload (device copies)."""
    w0 = ws[0]
    ts = None if w0.tensor_scale is None else torch.cat([w.tensor_scale for w in ws])
    scale = torch.cat([w.scale for w in ws])
    scale_dn = scale if w0.fmt != NVFP4 else torch.cat([w.scale_dn for w in ws])
    return QuantWeight(w0.N, w0.K, len(ws), w0.fmt, torch.cat([w.codes for w in ws]), scale, scale_dn, ts,
                       w0.scale_rule)


def version() -> str:
    return lib.sharq_version().decode()

"""Python binding of libmla_sparse.so (C ABI in include/mla_sparse.h).

Argument marshalling only: torch tensors are described to the library by
pointer, dtype, shape and strides, and the current HIP stream is passed
along.  Every step of the computation runs in the library's HIP kernels;
there is no fallback, and a missing library raises.
"""
from __future__ import annotations

import collections
import ctypes
import functools
import os
import struct

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmla_sparse.so")

DLAT, DPE, BLOCK, MAX_PARTS = 512, 64, 64, 64

MLA_OK = 0
MLA_ERR_INVALID_ARGUMENT = -1
MLA_ERR_UNSUPPORTED = -2
MLA_ERR_HIP = -3
MLA_ERR_OUT_OF_MEMORY = -4

DTYPE_BF16, DTYPE_FP8_E4M3FN, DTYPE_FP32, DTYPE_INT32, DTYPE_MXFP4 = 1, 2, 3, 4, 5
MX4_ROW = 272  # bytes of a 4-bit latent row: 256 of codes, 16 scale exponents

EXPORTS = ("mla_sparse_partial_attn", "mla_sparse_partial_attn_ex",
           "mla_sparse_partial_attn_tokens", "mla_merge_partials", "mla_merge_partials_ex",
           "mla_last_error", "mla_version", "mla_primitive_costs", "mla_fetch_gather",
           "mla_fetch_splice", "mla_sparse_partial_attn_noalloc", "mla_batch_slots", "mla_rope",
           "mla_cache_append", "mla_window_attn")


class MlaError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"status {status}: {msg}")
        self.status = status


class Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("ndim", ctypes.c_int32),
                ("shape", ctypes.c_int64 * 4), ("stride", ctypes.c_int64 * 4),
                ("block_scale", ctypes.c_void_p)]


class CostModel(ctypes.Structure):
    _fields_ = [("probe_us", ctypes.c_double), ("route_bw_gbs", ctypes.c_double),
                ("compute_us", ctypes.c_double), ("merge_us", ctypes.c_double),
                ("pull_bw_gbs", ctypes.c_double), ("splice_us", ctypes.c_double),
                ("prefill_us", ctypes.c_double), ("layers", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class CostCase(ctypes.Structure):
    _fields_ = [("mq", ctypes.c_int64), ("chunk_tokens", ctypes.c_int64),
                ("q_bytes", ctypes.c_int64), ("p_bytes", ctypes.c_int64),
                ("kv_bytes", ctypes.c_int64)]


class Cost(ctypes.Structure):
    _fields_ = [("route_us", ctypes.c_double), ("fetch_us", ctypes.c_double),
                ("local_us", ctypes.c_double), ("choice", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("wire_crossover_mq", ctypes.c_double),
                ("wire_saving", ctypes.c_double), ("congestion_bw_gbs", ctypes.c_double),
                ("splice_crossover_tokens", ctypes.c_double)]


PRIMITIVES = ("route", "fetch", "local")
# the constants the paper measured (Sections 4.3 and 5.1; c in [0.5, 1.5])
PAPER_COST_MODEL = dict(probe_us=16.0, route_bw_gbs=25.0, compute_us=0.0, merge_us=0.0,
                        pull_bw_gbs=25.0, splice_us=3000.0, prefill_us=1.0, layers=27)


class PartialOpts(ctypes.Structure):
    _fields_ = [("n_splits", ctypes.c_int32), ("row_tile", ctypes.c_int32),
                ("out_format", ctypes.c_int32), ("reserved", ctypes.c_int32 * 5)]


OUT_FP32, OUT_BF16_WIRE = 0, 1


class WindowOpts(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("n_sink", ctypes.c_int32), ("n_splits", ctypes.c_int32),
                ("out_format", ctypes.c_int32), ("row_tile", ctypes.c_int32),
                ("reserved", ctypes.c_int32 * 3)]


class RopeOpts(ctypes.Structure):
    _fields_ = [("rot_offset", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("pairing", ctypes.c_int32), ("scaling", ctypes.c_int32),
                ("inverse", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double),
                ("mscale", ctypes.c_double), ("orig_len", ctypes.c_int64)]


ROPE_SCALINGS = ("none", "linear", "yarn")


_lib = None


def load(path: str = LIB_PATH):
    """Load the library (once) and declare its entry points."""
    global _lib
    if _lib is not None and path == LIB_PATH:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run __graft_entry__.build() first")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER(Tensor)
    PP = ctypes.POINTER(P)
    vp = ctypes.c_void_p
    lib.mla_sparse_partial_attn.restype = ctypes.c_int
    lib.mla_sparse_partial_attn.argtypes = [P, P, P, P, P, P, ctypes.c_float, P, P, vp]
    lib.mla_sparse_partial_attn_ex.restype = ctypes.c_int
    lib.mla_sparse_partial_attn_ex.argtypes = [P, P, P, P, P, P, ctypes.c_float, P, P,
                                               ctypes.POINTER(PartialOpts), vp]
    lib.mla_sparse_partial_attn_tokens.restype = ctypes.c_int
    lib.mla_sparse_partial_attn_tokens.argtypes = lib.mla_sparse_partial_attn_ex.argtypes
    lib.mla_sparse_partial_attn_noalloc.restype = ctypes.c_int
    lib.mla_sparse_partial_attn_noalloc.argtypes = lib.mla_sparse_partial_attn_ex.argtypes
    lib.mla_merge_partials.restype = ctypes.c_int
    lib.mla_merge_partials.argtypes = [PP, PP, ctypes.c_int32, P, vp]
    lib.mla_merge_partials_ex.restype = ctypes.c_int
    lib.mla_merge_partials_ex.argtypes = [PP, PP, ctypes.c_int32, P, P, vp]
    lib.mla_fetch_gather.restype = ctypes.c_int
    lib.mla_fetch_gather.argtypes = [P, P, P, P, P, P, vp]
    lib.mla_fetch_splice.restype = ctypes.c_int
    lib.mla_fetch_splice.argtypes = [P, P, P, P, P, ctypes.c_int64, ctypes.c_int64,
                                     ctypes.c_float, ctypes.c_int32, vp]
    lib.mla_window_attn.restype = ctypes.c_int
    lib.mla_window_attn.argtypes = [P] * 7 + [ctypes.c_float, P, P, ctypes.POINTER(WindowOpts), vp]
    lib.mla_batch_slots.restype = ctypes.c_int
    lib.mla_batch_slots.argtypes = [P] * 9 + [vp]
    lib.mla_rope.restype = ctypes.c_int
    lib.mla_rope.argtypes = [P, P, P, ctypes.POINTER(RopeOpts), vp]
    lib.mla_cache_append.restype = ctypes.c_int
    lib.mla_cache_append.argtypes = [P] * 5 + [vp]
    lib.mla_primitive_costs.restype = ctypes.c_int
    lib.mla_primitive_costs.argtypes = [ctypes.POINTER(CostModel), ctypes.POINTER(CostCase),
                                        ctypes.POINTER(Cost)]
    lib.mla_last_error.restype = ctypes.c_char_p
    lib.mla_last_error.argtypes = []
    lib.mla_version.restype = ctypes.c_int32
    lib.mla_version.argtypes = []
    if path == LIB_PATH:
        _lib = lib
    return lib


_TORCH_DTYPES = {
    torch.bfloat16: DTYPE_BF16,
    torch.float32: DTYPE_FP32,
    torch.int32: DTYPE_INT32,
    torch.uint8: DTYPE_FP8_E4M3FN,
    torch.float8_e4m3fn: DTYPE_FP8_E4M3FN,
}


# mla_tensor_t packed field by field: data, dtype, ndim, shape[4], stride[4],
# block_scale (88 bytes, no padding on x86-64)
_PACK = struct.Struct("=Qii4q4qQ")
assert _PACK.size == ctypes.sizeof(Tensor)
_PAD = ((), (0,), (0, 0), (0, 0, 0), (0, 0, 0, 0))


def describe(t: torch.Tensor | None, block_scale: torch.Tensor | None = None) -> Tensor | None:
    """mla_tensor_t for a torch tensor (uint8 tensors are fp8-e4m3fn codes)."""
    if t is None:
        return None
    shape, stride = t.shape, t.stride()
    nd = len(shape)
    if nd > 4:
        raise ValueError("at most 4 dims")
    bs = 0
    if block_scale is not None:
        if block_scale.dtype != torch.float32 or not block_scale.is_contiguous():
            raise ValueError("block_scale must be contiguous float32")
        bs = block_scale.data_ptr()
    pad = _PAD[4 - nd]
    return Tensor.from_buffer_copy(_PACK.pack(t.data_ptr() if t.numel() else 0,
                                              _TORCH_DTYPES.get(t.dtype, 0), nd, *shape, *pad,
                                              *stride, *pad, bs))


def _describe_latent(t, block_scale=None):
    """describe() of a latent pool: a uint8 pool with rows of MX4_ROW bytes is
    a 4-bit one (MXFP4), with rows of 512 an fp8 one."""
    d = describe(t, block_scale)
    if t.dtype == torch.uint8 and t.dim() and t.shape[-1] == MX4_ROW:
        d.dtype = DTYPE_MXFP4
    return d


def _on_one_gpu(*tensors):
    """Raise ValueError unless every given tensor lives on one CUDA (HIP)
    device: the library reads and writes device memory only, and a host
    tensor's address handed to a kernel would fault.  Returns its index."""
    first = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"tensors must be on the GPU, got {t.device}")
        if first is None:
            first = t.get_device()
        elif t.get_device() != first:
            raise ValueError(f"tensors must be on one device, got {['cuda:%d' % first, str(t.device)]}")
    return first


def _on_current_gpu(*tensors, stream=None):
    """_on_one_gpu, and that device is the current one, on whose stream (or the
    given one, of the same device) the call goes, and in whose memory its
    workspace lies.  Returns its index."""
    dev = _on_one_gpu(*tensors)
    if dev != torch.cuda.current_device():
        raise ValueError(f"tensors are on cuda:{dev}, which is not the current device")
    at = getattr(stream, "device_index", dev)
    if at != dev:
        raise ValueError(f"tensors are on cuda:{dev}, the stream is on cuda:{at}")
    return dev


@functools.cache
def _several_gpus():
    return torch.cuda.device_count() > 1


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _check(lib, st):
    if st != MLA_OK:
        raise MlaError(st, lib.mla_last_error().decode())


def _ref(d):
    return ctypes.byref(d) if d is not None else None


class _Prepared:
    """One library call with its arguments fixed: the descriptors are built
    once and the tensors they point to are kept alive, so each call costs
    one foreign call (for serving loops that reuse static buffers)."""

    def __init__(self, fn, args, keep, result, device):
        self._fn, self._args, self._keep, self.result = fn, args, keep, result
        # (nothing to look at in each call where there is one device)
        self._device = device if _several_gpus() else None

    def __call__(self):
        if self._device is not None and torch.cuda.current_device() != self._device:
            raise ValueError(f"the call was prepared on cuda:{self._device}, which is not the current device")
        st = self._fn(*self._args)
        if st != MLA_OK:
            raise MlaError(st, load().mla_last_error().decode())
        return self.result


def _attn_outputs(R, q_lat, out_lat, out_lse, wire):
    _, Mq, H, _ = q_lat.shape
    if out_lat is None:
        out_lat = torch.empty((R, Mq, H, DLAT), dtype=torch.bfloat16 if wire else torch.float32,
                              device=q_lat.device)
    if out_lse is None:
        out_lse = torch.empty((R, Mq, H, 2) if wire else (R, Mq, H), dtype=torch.float32,
                              device=q_lat.device)
    return out_lat, out_lse


def _partial_args(q_lat, q_pe, ckv_pool, kpe_pool, chunk_block_table, sel_block_ids, scale,
                  out_lat, out_lse, ckv_scale, kpe_scale, n_splits, row_tile, stream, wire=False):
    R = chunk_block_table.shape[0]  # jobs; q may hold fewer rows (R_q dividing R)
    out_lat, out_lse = _attn_outputs(R, q_lat, out_lat, out_lse, wire)
    dev = _on_current_gpu(q_lat, q_pe, ckv_pool, kpe_pool, chunk_block_table, sel_block_ids, out_lat,
                          out_lse, ckv_scale, kpe_scale, stream=stream)
    opts = PartialOpts()
    opts.n_splits = int(n_splits)
    opts.row_tile = int(row_tile)
    opts.out_format = OUT_BF16_WIRE if wire else OUT_FP32
    descs = (describe(q_lat), describe(q_pe), _describe_latent(ckv_pool, ckv_scale),
             describe(kpe_pool, kpe_scale), describe(chunk_block_table), describe(sel_block_ids))
    outs = (describe(out_lat), describe(out_lse))
    args = tuple(_ref(d) for d in descs) + (ctypes.c_float(scale),) + \
        tuple(_ref(d) for d in outs) + (ctypes.byref(opts), _stream(stream))
    keep = (descs, outs, opts, q_lat, q_pe, ckv_pool, kpe_pool, chunk_block_table,
            sel_block_ids, ckv_scale, kpe_scale)
    return args, keep, (out_lat, out_lse), dev


def _partial_fn(lib, tokens, no_alloc):
    if tokens and no_alloc:
        raise ValueError("the allocation-free entry point takes block selections only")
    if no_alloc:
        return lib.mla_sparse_partial_attn_noalloc
    return lib.mla_sparse_partial_attn_tokens if tokens else lib.mla_sparse_partial_attn_ex


def prepare_partial(q_lat, q_pe, ckv_pool, kpe_pool, chunk_block_table, sel_block_ids, scale,
                    out_lat=None, out_lse=None, ckv_scale=None, kpe_scale=None, n_splits=0,
                    row_tile=0, stream=None, tokens=False, no_alloc=False, wire=False):
    """sparse_partial_attn with every argument fixed, the stream included
    (the current one when None); calling the result launches the work and
    returns (out_lat, out_lse)."""
    args, keep, result, dev = _partial_args(q_lat, q_pe, ckv_pool, kpe_pool, chunk_block_table,
                                            sel_block_ids, scale, out_lat, out_lse, ckv_scale,
                                            kpe_scale, n_splits, row_tile, stream, wire)
    lib = load()
    return _Prepared(_partial_fn(lib, tokens, no_alloc), args, keep, result, dev)


def sparse_partial_attn(q_lat, q_pe, ckv_pool, kpe_pool, chunk_block_table, sel_block_ids,
                        scale, out_lat=None, out_lse=None, ckv_scale=None, kpe_scale=None,
                        n_splits=0, row_tile=0, stream=None, tokens=False, no_alloc=False,
                        wire=False):
    """Partial attention of each job's Mq x H rows over its selected blocks,
    or with tokens=True over its selected single tokens (sel_block_ids then
    holds logical token ids, block * 64 + t).  no_alloc=True calls the
    allocation-free entry point (split-K partials in the library's static
    scratch array; block selections only).  wire=True asks for the bf16
    wire form of Section 3.2.

    Returns (out_lat fp32 [R, Mq, H, 512], out_lse fp32 [R, Mq, H]), or with
    wire=True (out_lat bf16 [R, Mq, H, 512], (m, l) pairs fp32 [R, Mq, H, 2]).
    """
    lib = load()
    args, _keep, result, _ = _partial_args(q_lat, q_pe, ckv_pool, kpe_pool, chunk_block_table,
                                           sel_block_ids, scale, out_lat, out_lse, ckv_scale,
                                           kpe_scale, n_splits, row_tile, stream, wire)
    _check(lib, _partial_fn(lib, tokens, no_alloc)(*args))
    return result


def prepare_window(q_lat, q_pe, ckv_pool, kpe_pool, block_table, seq_lens, scale, window=0, n_sink=0,
                   q_lens=None, out_lat=None, out_lse=None, ckv_scale=None, kpe_scale=None,
                   n_splits=0, stream=None, wire=False, row_tile=0):
    """window_attn with every argument fixed (see prepare_partial)."""
    out = _attn_outputs(block_table.shape[0], q_lat, out_lat, out_lse, wire)
    dev = _on_current_gpu(q_lat, q_pe, ckv_pool, kpe_pool, block_table, seq_lens, q_lens, *out, ckv_scale,
                          kpe_scale, stream=stream)
    o = WindowOpts(int(window), int(n_sink), int(n_splits), OUT_BF16_WIRE if wire else OUT_FP32,
                   int(row_tile))
    d = (describe(q_lat), describe(q_pe), _describe_latent(ckv_pool, ckv_scale),
         describe(kpe_pool, kpe_scale), describe(block_table), describe(seq_lens), describe(q_lens))
    do = tuple(describe(t) for t in out)
    args = (*[_ref(x) for x in d], ctypes.c_float(scale), *[_ref(x) for x in do], ctypes.byref(o),
            _stream(stream))
    keep = (d, do, o, q_lat, q_pe, ckv_pool, kpe_pool, block_table, seq_lens, q_lens, ckv_scale,
            kpe_scale)
    return _Prepared(load().mla_window_attn, args, keep, out, dev)


def window_attn(q_lat, q_pe, ckv_pool, kpe_pool, block_table, seq_lens, scale, window=0, n_sink=0,
                q_lens=None, out_lat=None, out_lse=None, ckv_scale=None, kpe_scale=None, n_splits=0,
                stream=None, wire=False, row_tile=0):
    """Attention of each request's last q_lens[b] tokens (default: all Mq query
    rows) over its paged sequence of seq_lens[b] tokens, each row seeing the
    last `window` tokens up to its own (0: all) and the first n_sink.  Pools
    are bf16, fp8 (uint8 with scales) or 4-bit (uint8 rows of MX4_ROW bytes,
    the RoPE pool bf16).  Returns partials as sparse_partial_attn does, in
    either form, for merge_partials or as they are."""
    return prepare_window(q_lat, q_pe, ckv_pool, kpe_pool, block_table, seq_lens, scale, window,
                          n_sink, q_lens, out_lat, out_lse, ckv_scale, kpe_scale, n_splits, stream,
                          wire, row_tile)()


def fetch_gather(ckv_pool, kpe_pool, chunk_block_table, sel_token_ids, out_ckv=None,
                 out_kpe=None, stream=None):
    """FETCH's scattered gather: the selected tokens of every layer, in slot
    order, as contiguous bf16 [L, K, 512] / [L, K, 64] (zero rows for empty
    slots).  Pools are [L, P, 64, 512] / [L, P, 64, 64] bf16, or the latent one
    [L, P, 64, 272] in 4 bits (uint8), whose values are exact in bf16."""
    L = ckv_pool.shape[0]
    K = sel_token_ids.shape[0]
    if out_ckv is None:
        out_ckv = torch.empty((L, K, DLAT), dtype=torch.bfloat16, device=ckv_pool.device)
    if out_kpe is None:
        out_kpe = torch.empty((L, K, DPE), dtype=torch.bfloat16, device=ckv_pool.device)
    _on_current_gpu(ckv_pool, kpe_pool, chunk_block_table, sel_token_ids, out_ckv, out_kpe, stream=stream)
    lib = load()
    d = [_describe_latent(ckv_pool)]
    d += [describe(t) for t in (kpe_pool, chunk_block_table, sel_token_ids, out_ckv, out_kpe)]
    _check(lib, lib.mla_fetch_gather(*[_ref(x) for x in d], _stream(stream)))
    return out_ckv, out_kpe


def fetch_splice(chunk_ckv, chunk_kpe, ckv_pool, kpe_pool, block_table, dst_start, delta,
                 rope_base=10000.0, pairing=0, stream=None):
    """FETCH's splice: write the chunk [L, n, 512] / [L, n, 64] into the
    paged pools at positions dst_start .. dst_start + n - 1 of the sequence
    that block_table maps, its RoPE pairs turned by delta positions
    (pairing 0: dims (2i, 2i+1), 1: dims (i, i+32))."""
    _on_current_gpu(chunk_ckv, chunk_kpe, ckv_pool, kpe_pool, block_table, stream=stream)
    lib = load()
    d = [describe(t) for t in (chunk_ckv, chunk_kpe, ckv_pool, kpe_pool, block_table)]
    _check(lib, lib.mla_fetch_splice(*[_ref(x) for x in d], int(dst_start), int(delta),
                                     float(rope_base), int(pairing), _stream(stream)))


SlotPlan = collections.namedtuple("SlotPlan", "slots positions seq_lens starts info")


def prepare_batch_slots(cached_lens, new_lens, free_blocks, block_table, n_tokens=None, slots=None,
                        positions=None, seq_lens=None, starts=None, info=None, stream=None):
    """batch_slots with every argument fixed (see prepare_partial)."""
    B, dev = cached_lens.shape[0], cached_lens.device
    if slots is None:
        if n_tokens is None:
            raise ValueError("give n_tokens (the most new tokens of a call) or slots")
        slots = torch.empty(n_tokens, dtype=torch.int32, device=dev)

    def out(t, n):
        return torch.empty(n, dtype=torch.int32, device=dev) if t is None else t
    plan = SlotPlan(slots, out(positions, slots.shape[0]), out(seq_lens, B), out(starts, B + 1), out(info, 4))
    gpu = _on_current_gpu(cached_lens, new_lens, free_blocks, block_table, *plan, stream=stream)
    keep = (cached_lens, new_lens, free_blocks, block_table)
    d = [describe(t) for t in (*keep, *plan)]
    return _Prepared(load().mla_batch_slots, (*[_ref(x) for x in d], _stream(stream)), (d, keep), plan, gpu)


def batch_slots(cached_lens, new_lens, free_blocks, block_table, n_tokens=None, slots=None,
                positions=None, seq_lens=None, starts=None, info=None, stream=None):
    """Block tables and slot maps of a batch from its lengths, on the GPU:
    extends block_table [B, NB] in place with blocks of free_blocks, and
    returns SlotPlan(slots, positions, seq_lens, starts, info) for the new
    tokens packed request after request (see mla_batch_slots in the header).
    n_tokens, or the length of a given slots, is the most tokens it holds."""
    return prepare_batch_slots(cached_lens, new_lens, free_blocks, block_table, n_tokens, slots,
                               positions, seq_lens, starts, info, stream)()


def prepare_rope(x, positions, out=None, rot_offset=0, rot_dim=None, pairing=0, base=10000.0,
                 scaling="none", factor=1.0, orig_len=0, beta_fast=32.0, beta_slow=1.0, mscale=1.0,
                 inverse=False, stream=None):
    """rope with every argument fixed (see prepare_partial).  No gradients go
    through the call: x must not require them where they are recorded."""
    if x.dim() != 3:
        raise ValueError("x must be [T, H, D]")
    if torch.is_grad_enabled() and (x.requires_grad or (out is not None and out.requires_grad)):
        raise ValueError("gradients go through rope(x, ...) without out only: detach x, or call under no_grad")
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dev = _on_current_gpu(x, positions, out, stream=stream)
    o = RopeOpts(int(rot_offset), int(x.shape[2] - rot_offset if rot_dim is None else rot_dim),
                 int(pairing), ROPE_SCALINGS.index(scaling), int(bool(inverse)), 0, float(base),
                 float(factor), float(beta_fast), float(beta_slow), float(mscale), int(orig_len))
    d = [describe(t) for t in (x, positions, out)]
    return _Prepared(load().mla_rope, (*[_ref(t) for t in d], ctypes.byref(o), _stream(stream)),
                     (d, o, x, positions), out, dev)


class _Rope(torch.autograd.Function):
    """rope with its gradient, the transposed map: a rope that turns back."""

    @staticmethod
    def forward(ctx, x, positions, opts, inverse, stream):
        ctx.save_for_backward(positions)
        ctx.opts, ctx.inverse = opts, inverse
        return prepare_rope(x, positions, None, *opts, inverse, stream)()

    @staticmethod
    def backward(ctx, g):
        positions, = ctx.saved_tensors
        # (the gradient of a sum is one number under strides of 0)
        g = g if g.stride(2) == 1 else g.contiguous()
        return rope(g, positions, None, *ctx.opts, not ctx.inverse), None, None, None, None


def rope(x, positions, out=None, rot_offset=0, rot_dim=None, pairing=0, base=10000.0,
         scaling="none", factor=1.0, orig_len=0, beta_fast=32.0, beta_slow=1.0, mscale=1.0,
         inverse=False, stream=None):
    """Rotary positions of x [T, H, D] (bf16 or fp32): dims rot_offset ..
    rot_offset + rot_dim - 1 (default: to the end) of row t turn by
    positions[t], the others are copied.  pairing 0: dims (2i, 2i+1), 1: (i,
    i + rot_dim/2); scaling "none", "linear" (factor) or "yarn" (factor,
    orig_len, beta_fast, beta_slow); out may be x.  inverse=True is the
    transpose of the map, which takes gradients of out to gradients of x: an x
    that requires them gets them (the one call here that records any), without
    out.  A graph that captures the backward captures its forward too, and takes
    the gradients by torch.autograd.grad."""
    opts = (rot_offset, rot_dim, pairing, base, scaling, factor, orig_len, beta_fast, beta_slow, mscale)
    if out is None and torch.is_grad_enabled() and x.requires_grad:
        return _Rope.apply(x, positions, opts, inverse, stream)
    return prepare_rope(x, positions, out, *opts, inverse, stream)()


def prepare_cache_append(ckv, kpe, slots, ckv_pool, kpe_pool, stream=None):
    """cache_append with every argument fixed (see prepare_partial)."""
    dev = _on_current_gpu(ckv, kpe, slots, ckv_pool, kpe_pool, stream=stream)
    d = [describe(ckv), describe(kpe), describe(slots), _describe_latent(ckv_pool), describe(kpe_pool)]
    return _Prepared(load().mla_cache_append, (*[_ref(t) for t in d], _stream(stream)),
                     (d, ckv, kpe, slots), (ckv_pool, kpe_pool), dev)


def cache_append(ckv, kpe, slots, ckv_pool, kpe_pool, stream=None):
    """Writes new tokens [T, 512] / [T, 64] (bf16) into the pools at slots
    (block * 64 + row; others than the pool's are skipped): a bf16 latent pool
    [P, 64, 512] as they are, a 4-bit one [P, 64, 272] (uint8) as E2M1 codes
    under a power of two per 32 columns.  Returns the pools."""
    return prepare_cache_append(ckv, kpe, slots, ckv_pool, kpe_pool, stream)()


def primitive_costs(mq, chunk_tokens, q_bytes=1152, p_bytes=1032, kv_bytes=1152, **model):
    """ROUTE / FETCH / LOCAL costs of one (chunk, request) case from the
    closed-form model (host arithmetic in the library).  `model` overrides
    fields of PAPER_COST_MODEL.  Returns a dict of the mla_cost_t fields,
    with `choice` as a primitive name."""
    lib = load()
    m = CostModel(**{**PAPER_COST_MODEL, **model})
    c = CostCase(mq, chunk_tokens, q_bytes, p_bytes, kv_bytes)
    out = Cost()
    _check(lib, lib.mla_primitive_costs(ctypes.byref(m), ctypes.byref(c), ctypes.byref(out)))
    res = {f: getattr(out, f) for f, _ in Cost._fields_ if f != "reserved"}
    res["choice"] = PRIMITIVES[res["choice"]]
    return res


def _merge_args(parts_lat, parts_lse, out, out_lse, stream):
    n = len(parts_lat)
    if n != len(parts_lse):
        raise ValueError("parts_lat and parts_lse differ in length")
    want_lse = out_lse is not None
    if out is None:  # fp32 whatever form the parts take
        out = torch.empty(parts_lat[0].shape, dtype=torch.float32, device=parts_lat[0].device)
    if out_lse is True:
        out_lse = torch.empty(parts_lse[0].shape[:3], dtype=torch.float32,
                              device=parts_lse[0].device)
    dev = _on_current_gpu(*parts_lat, *parts_lse, out, out_lse if want_lse else None, stream=stream)
    d_lat = [describe(t) for t in parts_lat]
    d_lse = [describe(t) for t in parts_lse]
    arr_lat = (ctypes.POINTER(Tensor) * max(n, 1))(*[ctypes.pointer(d) for d in d_lat])
    arr_lse = (ctypes.POINTER(Tensor) * max(n, 1))(*[ctypes.pointer(d) for d in d_lse])
    d_out = describe(out)
    d_out_lse = describe(out_lse) if want_lse else None
    args = (arr_lat, arr_lse, n, _ref(d_out), _ref(d_out_lse), _stream(stream))
    keep = (d_lat, d_lse, d_out, d_out_lse, list(parts_lat), list(parts_lse))
    return args, keep, ((out, out_lse) if want_lse else out), dev


def prepare_merge(parts_lat, parts_lse, out=None, out_lse=None, stream=None):
    """merge_partials with every argument fixed (see prepare_partial)."""
    args, keep, result, dev = _merge_args(parts_lat, parts_lse, out, out_lse, stream)
    return _Prepared(load().mla_merge_partials_ex, args, keep, result, dev)


def merge_partials(parts_lat, parts_lse, out=None, out_lse=None, stream=None):
    """LSE merge of partials (lists of [B, Mq, H, 512] / [B, Mq, H] fp32, or
    of wire-form parts: [B, Mq, H, 512] bf16 / [B, Mq, H, 2] (m, l) fp32).

    Returns out (and the merged lse when out_lse is given or requested by
    passing out_lse=True)."""
    lib = load()
    args, _keep, result, _ = _merge_args(parts_lat, parts_lse, out, out_lse, stream)
    _check(lib, lib.mla_merge_partials_ex(*args))
    return result

"""Thin ctypes binding of the C ABI in include/mv.h (libmv.so).

Argument marshalling only: every step of the vote step runs in the library's
HIP kernels.  PyTorch tensors supply device memory and the stream.  There is no
fallback: if libmv.so has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmv.so")

MV_OK, MV_ERR_INVALID_ARG, MV_ERR_UNSUPPORTED, MV_ERR_ALLOC, MV_ERR_DEVICE, MV_ERR_STATE = range(6)
MV_F32, MV_BF16 = 0, 1
MV_REDUCE_MEAN, MV_REDUCE_SUM = 0, 1
MV_FLAG_ADD_DROP = 1
MV_NORM_L2, MV_NORM_MAX = 0, 1

# every symbol include/mv.h declares
ABI_SYMBOLS = (
    "mv_workspace_bytes", "mv_begin", "mv_vote_step", "mv_ad_vote_step", "mv_rs_vote_step", "mv_end", "mv_release", "mv_status_string",
    "mv_kernel_count", "mv_kernel_name", "mv_set_profiling", "mv_set_spin_limit", "mv_step_kernel_ms",
    "mv_last_step_row_stats", "mv_probe_copy",
    "mv_codec_stream_bits", "mv_codec_scratch_bytes", "mv_codec_encode", "mv_codec_decode", "mv_codec_decode_static",
    "mv_quant_scratch_bytes", "mv_quant_encode", "mv_quant_decode",
    "mv_clip_workspace_bytes", "mv_clip_begin", "mv_clip_bind", "mv_clip_norms", "mv_clip_grads",
    "mv_clip_set_spin_limit", "mv_clip_end", "mv_clip_release",
    "mv_mx_row_words", "mv_mx_row_scales", "mv_mx_encode", "mv_mx_encode_t", "mv_mx_decode", "mv_mx_aggregate",
    "mv_mx_product_scratch_bytes", "mv_mx_product", "mv_mx_linear_scratch_bytes", "mv_mx_linear",
    "mv_mx_linear_grad_scratch_bytes", "mv_mx_linear_grad",
    "mv_f8_row_bytes", "mv_f8_row_scales", "mv_f8_encode", "mv_f8_encode_t", "mv_f8_decode",
    "mv_f8_product_scratch_bytes", "mv_f8_product", "mv_f8_linear_scratch_bytes", "mv_f8_linear",
    "mv_f8_linear_grad_scratch_bytes", "mv_f8_linear_grad",
    "mv_layernorm_forward", "mv_layernorm_scratch_bytes", "mv_layernorm_backward",
    "mv_distill_scratch_bytes", "mv_distill_loss", "mv_distill_grad",
)


class mv_config(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("device", ctypes.c_int32),
        ("n_workers", ctypes.c_int32),
        ("grad_dtype", ctypes.c_int32),
        ("d", ctypes.c_int64),
        ("k", ctypes.c_int64),
        ("reduce", ctypes.c_int32),
        ("flags", ctypes.c_int32),
        ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t),
    ]


class mv_clip_tensor(ctypes.Structure):
    _fields_ = [
        ("src", ctypes.c_void_p),
        ("dst", ctypes.c_void_p),
        ("numel", ctypes.c_int64),
        ("group", ctypes.c_int32),
        ("src_dtype", ctypes.c_int16),
        ("dst_dtype", ctypes.c_int16),
    ]


class mv_clip_config(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("device", ctypes.c_int32),
        ("n_groups", ctypes.c_int32),
        ("norm", ctypes.c_int32),
        ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t),
    ]


class MvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (where, status_string(status), status))


_lib: Optional[ctypes.CDLL] = None


def load() -> ctypes.CDLL:
    """Loads libmv.so (built by paper_2011_06495_amd.build / __graft_entry__.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            "%s is missing: build it first (python -m paper_2011_06495_amd.build); "
            "there is no CPU fallback" % LIB_PATH)
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u32p = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.POINTER(ctypes.c_uint32)
    L.mv_workspace_bytes.argtypes = [ctypes.POINTER(mv_config)]
    L.mv_workspace_bytes.restype = ctypes.c_size_t
    L.mv_begin.argtypes = [ctypes.POINTER(mv_config), ctypes.POINTER(vp)]
    L.mv_begin.restype = i32
    L.mv_vote_step.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, vp, vp]
    L.mv_vote_step.restype = i32
    L.mv_ad_vote_step.argtypes = [vp, vp, i64, vp, i64, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp]
    L.mv_ad_vote_step.restype = i32
    L.mv_rs_vote_step.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp]
    L.mv_rs_vote_step.restype = i32
    L.mv_end.argtypes = [vp]
    L.mv_end.restype = i32
    L.mv_release.argtypes = [vp]
    L.mv_release.restype = None
    L.mv_status_string.argtypes = [i32]
    L.mv_status_string.restype = ctypes.c_char_p
    L.mv_kernel_count.argtypes = []
    L.mv_kernel_count.restype = i32
    L.mv_kernel_name.argtypes = [i32]
    L.mv_kernel_name.restype = ctypes.c_char_p
    L.mv_set_profiling.argtypes = [vp, i32]
    L.mv_set_profiling.restype = i32
    L.mv_set_spin_limit.argtypes = [vp, ctypes.c_uint32]
    L.mv_set_spin_limit.restype = i32
    L.mv_step_kernel_ms.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_float), i32]
    L.mv_step_kernel_ms.restype = i32
    L.mv_last_step_row_stats.argtypes = [vp, u32p, u32p, u32p]
    L.mv_last_step_row_stats.restype = i32
    u64 = ctypes.c_uint64
    L.mv_codec_stream_bits.argtypes = [i64, i64, i64]
    L.mv_codec_stream_bits.restype = u64
    L.mv_codec_scratch_bytes.argtypes = [u64, i32]
    L.mv_codec_scratch_bytes.restype = ctypes.c_size_t
    L.mv_codec_encode.argtypes = [vp, i64, vp, i64, i64, i32, i64, i64, vp, i64, vp, vp]
    L.mv_codec_encode.restype = i32
    L.mv_codec_decode.argtypes = [vp, i64, vp, u64, i32, i64, i64, vp, i64, i64, vp, vp, ctypes.c_size_t, vp]
    L.mv_codec_decode.restype = i32
    L.mv_codec_decode_static.argtypes = [vp, i64, vp, u64, i32, i64, i64, vp, i64, i64, vp, vp]
    L.mv_codec_decode_static.restype = i32
    L.mv_quant_scratch_bytes.argtypes = [i64, i32, i32]
    L.mv_quant_scratch_bytes.restype = ctypes.c_size_t
    L.mv_quant_encode.argtypes = [vp, i64, i64, i32, i32, vp, i64, vp, vp, ctypes.c_size_t, vp]
    L.mv_quant_encode.restype = i32
    L.mv_quant_decode.argtypes = [vp, i64, i64, i32, i32, vp, vp, i64, vp]
    L.mv_quant_decode.restype = i32
    sz, f32 = ctypes.c_size_t, ctypes.c_float
    L.mv_clip_workspace_bytes.argtypes = [ctypes.POINTER(mv_clip_config), vp, i64]
    L.mv_clip_workspace_bytes.restype = sz
    L.mv_clip_begin.argtypes = [ctypes.POINTER(mv_clip_config), vp, i64, ctypes.POINTER(vp)]
    L.mv_clip_bind.argtypes = [vp, vp, vp, vp]
    L.mv_clip_norms.argtypes = [vp, vp, vp]
    L.mv_clip_grads.argtypes = [vp, f32, vp, vp, vp]
    L.mv_clip_set_spin_limit.argtypes = [vp, ctypes.c_uint32]
    L.mv_clip_end.argtypes = [vp]
    L.mv_clip_release.argtypes = [vp]
    L.mv_clip_release.restype = None
    L.mv_mx_row_words.argtypes = [i64]
    L.mv_mx_row_words.restype = i64
    L.mv_mx_row_scales.argtypes = [i64]
    L.mv_mx_row_scales.restype = i64
    L.mv_mx_encode.argtypes = [vp, i32, i64, i64, i64, vp, i64, vp, i64, vp, i64, vp]
    L.mv_mx_encode_t.argtypes = [vp, i32, i64, i64, i64, vp, i64, vp, i64, vp]
    L.mv_mx_decode.argtypes = [vp, i64, vp, i64, i64, i64, vp, i32, i64, vp]
    L.mv_mx_aggregate.argtypes = [vp, i64, vp, i64, i64, i64, vp, vp, vp]
    L.mv_f8_row_bytes.argtypes = [i64]
    L.mv_f8_row_bytes.restype = i64
    L.mv_f8_row_scales.argtypes = [i64]
    L.mv_f8_row_scales.restype = i64
    L.mv_f8_encode.argtypes = [vp, i32, i64, i64, i64, vp, i64, vp, i64, vp]
    L.mv_f8_encode_t.argtypes = [vp, i32, i64, i64, i64, vp, i64, vp, i64, vp]
    L.mv_f8_decode.argtypes = [vp, i64, vp, i64, i64, i64, vp, i32, i64, vp]
    for f in (L.mv_mx_product_scratch_bytes, L.mv_mx_linear_scratch_bytes, L.mv_mx_linear_grad_scratch_bytes,
              L.mv_f8_product_scratch_bytes, L.mv_f8_linear_scratch_bytes, L.mv_f8_linear_grad_scratch_bytes):
        f.argtypes = [i64, i64, i64]
        f.restype = sz
    L.mv_mx_product.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, i64, i64, i64, vp, i32, i64, vp, sz, vp]
    L.mv_mx_linear.argtypes = [vp, i32, i64, vp, i64, vp, i64, i64, i64, i64, vp, i32, i64, vp, sz, vp]
    L.mv_mx_linear_grad.argtypes = [vp, i64, vp, i64, i32, vp, i64, vp, i64, i64, i64, i64, vp, i32, i64, vp, i32, i64,
                                    vp, sz, vp]
    L.mv_f8_product.argtypes, L.mv_f8_linear.argtypes = L.mv_mx_product.argtypes, L.mv_mx_linear.argtypes
    L.mv_f8_linear_grad.argtypes = L.mv_mx_linear_grad.argtypes
    L.mv_layernorm_forward.argtypes = [vp, i32, i64, i64, i64, vp, vp, i32, f32, vp, i32, i64, vp, vp, vp]
    L.mv_layernorm_backward.argtypes = [vp, i64, vp, i64, i32, i64, i64, vp, i32, vp, vp, vp, i32, i64, vp, vp, vp, sz, vp]
    listed = [vp, i32, i64, i64, i64, vp, i64, vp, i32, i64, i64, vp, f32, f32, f32]
    L.mv_distill_loss.argtypes = listed + [vp, vp, vp, vp, i32, i64, vp, sz, vp]
    L.mv_distill_grad.argtypes = listed + [vp, vp, vp, i32, i64, vp]
    for f in (L.mv_layernorm_scratch_bytes, L.mv_distill_scratch_bytes):
        f.argtypes = [i64, i64]
        f.restype = sz
    for f in (L.mv_f8_encode, L.mv_f8_encode_t, L.mv_f8_decode, L.mv_f8_product, L.mv_f8_linear, L.mv_f8_linear_grad,
              L.mv_layernorm_forward, L.mv_layernorm_backward, L.mv_distill_loss, L.mv_distill_grad):
        f.restype = i32
    for f in (L.mv_clip_begin, L.mv_clip_bind, L.mv_clip_norms, L.mv_clip_grads, L.mv_clip_set_spin_limit, L.mv_clip_end, L.mv_mx_encode,
              L.mv_mx_encode_t, L.mv_mx_decode, L.mv_mx_aggregate, L.mv_mx_product, L.mv_mx_linear, L.mv_mx_linear_grad):
        f.restype = i32
    L.mv_probe_copy.argtypes = [vp, vp, ctypes.c_size_t, vp]
    L.mv_probe_copy.restype = i32
    _lib = L
    return L


def status_string(status: int) -> str:
    return load().mv_status_string(int(status)).decode()


def make_config(n_workers: int, d: int, k: int, grad_dtype: int = MV_F32, reduce: int = MV_REDUCE_MEAN,
                device: int = 0, workspace: int = 0, workspace_bytes: int = 0, flags: int = 0) -> mv_config:
    return mv_config(ctypes.sizeof(mv_config), device, n_workers, grad_dtype, d, k, reduce, flags,
                     workspace or None, workspace_bytes)


def mv_workspace_bytes(cfg: mv_config) -> int:
    return int(load().mv_workspace_bytes(ctypes.byref(cfg)))


def mv_begin(cfg: mv_config) -> int:
    """Returns the context handle (an integer address); raises MvError."""
    h = ctypes.c_void_p()
    st = load().mv_begin(ctypes.byref(cfg), ctypes.byref(h))
    if st != MV_OK:
        raise MvError(st, "mv_begin")
    return h.value


def _dev_ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


_raw_stream = None      # torch's own getter of the current stream's handle, once torch is there


def _stream_handle(stream, t) -> int:
    """The hipStream_t of `stream` (a torch.cuda.Stream), or of the current stream of t's device.
    The short calls of this library take a few microseconds on the GPU, less than building a
    torch.cuda.Stream object and the rest of a call took on the host (a loop of mv_quant_decode
    calls: 7.0 us each, 5.0 us so)."""
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    device = t.get_device()
    if device < 0:                       # not on a GPU: torch's own error
        import torch
        return torch.cuda.current_stream(t.device).cuda_stream
    if _raw_stream is None:
        import torch
        _raw_stream = torch._C._cuda_getCurrentRawStream
    return _raw_stream(device)


def mv_vote_step(ctx: int, grads, err, worker_idx, votes, mask_idx, agg_vals, stream=None,
                 ld_g: Optional[int] = None, ld_e: Optional[int] = None) -> None:
    """Enqueues one vote step on `stream` (a torch.cuda.Stream; None = torch's
    current stream).  Tensors are torch device tensors; `grads` and `err` are
    2-D with unit column stride (the row stride is taken from the tensor unless
    given).  worker_idx and votes may be None."""
    st = load().mv_vote_step(
        ctx, _dev_ptr(grads), grads.stride(0) if ld_g is None else ld_g,
        _dev_ptr(err), err.stride(0) if ld_e is None else ld_e,
        _dev_ptr(worker_idx), _dev_ptr(votes), _dev_ptr(mask_idx), _dev_ptr(agg_vals),
        _stream_handle(stream, err))
    if st != MV_OK:
        raise MvError(st, "mv_vote_step")


def mv_rs_vote_step(ctx: int, grads, err, rand_exp, worker_idx, votes, mask_idx, agg_vals, stream=None,
                    ld_g: Optional[int] = None, ld_e: Optional[int] = None) -> None:
    """Enqueues one step of majority voting with random selection: as mv_vote_step,
    the mask drawn in proportion to the votes with the caller's Exp(1) numbers
    `rand_exp` (d float32 on the device)."""
    st = load().mv_rs_vote_step(
        ctx, _dev_ptr(grads), grads.stride(0) if ld_g is None else ld_g,
        _dev_ptr(err), err.stride(0) if ld_e is None else ld_e, _dev_ptr(rand_exp),
        _dev_ptr(worker_idx), _dev_ptr(votes), _dev_ptr(mask_idx), _dev_ptr(agg_vals),
        _stream_handle(stream, err))
    if st != MV_OK:
        raise MvError(st, "mv_rs_vote_step")


def mv_ad_vote_step(ctx: int, grads, err, k_ad: int, vote_bits, msum, add_idx, drop_idx, counts, mask_idx,
                    agg_vals, stream=None, ld_g: Optional[int] = None, ld_e: Optional[int] = None) -> None:
    """Enqueues one add-drop vote step (Algorithm 2).  vote_bits: N x ld_bits int32
    device tensor (the standing votes' bitmaps), msum: uint8 device tensor."""
    st = load().mv_ad_vote_step(
        ctx, _dev_ptr(grads), grads.stride(0) if ld_g is None else ld_g,
        _dev_ptr(err), err.stride(0) if ld_e is None else ld_e, int(k_ad),
        _dev_ptr(vote_bits), vote_bits.stride(0), _dev_ptr(msum), _dev_ptr(add_idx), _dev_ptr(drop_idx),
        _dev_ptr(counts), _dev_ptr(mask_idx), _dev_ptr(agg_vals), _stream_handle(stream, err))
    if st != MV_OK:
        raise MvError(st, "mv_ad_vote_step")


def mv_end(ctx: int) -> None:
    st = load().mv_end(ctx)
    if st != MV_OK:
        raise MvError(st, "mv_end")


def mv_release(ctx: int) -> None:
    load().mv_release(ctx)


def kernel_names():
    L = load()
    return [L.mv_kernel_name(i).decode() for i in range(L.mv_kernel_count())]


def mv_set_profiling(ctx: int, level: int) -> None:
    st = load().mv_set_profiling(ctx, level)
    if st != MV_OK:
        raise MvError(st, "mv_set_profiling")


def mv_set_spin_limit(ctx: int, polls: int) -> None:
    st = load().mv_set_spin_limit(ctx, polls)
    if st != MV_OK:
        raise MvError(st, "mv_set_spin_limit")


def mv_step_kernel_ms(ctx: int, steps_back: int = 0):
    n = load().mv_kernel_count()
    buf = (ctypes.c_float * n)()
    st = load().mv_step_kernel_ms(ctx, steps_back, buf, n)
    if st != MV_OK:
        raise MvError(st, "mv_step_kernel_ms")
    return list(buf)


def mv_last_step_row_stats(ctx: int, n_workers: int):
    a, b, c = ((ctypes.c_uint32 * n_workers)() for _ in range(3))
    st = load().mv_last_step_row_stats(ctx, a, b, c)
    if st != MV_OK:
        raise MvError(st, "mv_last_step_row_stats")
    return list(a), list(b), list(c)


def mv_probe_copy(dst, src, stream=None) -> None:
    """Plain streaming copy src -> dst (torch device tensors of equal byte size)."""
    nbytes = src.numel() * src.element_size()
    assert dst.numel() * dst.element_size() == nbytes
    st = load().mv_probe_copy(dst.data_ptr(), src.data_ptr(), nbytes, _stream_handle(stream, src))
    if st != MV_OK:
        raise MvError(st, "mv_probe_copy")


def mv_codec_stream_bits(n: int, d: int, block_len: int) -> int:
    return int(load().mv_codec_stream_bits(n, d, block_len))


def mv_codec_scratch_bytes(max_bits: int, rows: int) -> int:
    return int(load().mv_codec_scratch_bytes(max_bits, rows))


def mv_codec_encode(idx, n: int, d: int, block_len: int, streams, n_bits, counts=None, counts_stride: int = 1,
                    stream=None) -> None:
    """idx: rows x ld int32 device tensor of ascending coordinates; streams: rows x ld_words
    int32 device tensor (out); n_bits: rows int64 device tensor (out); counts: optional
    int32 device tensor with the rows' lengths at stride counts_stride."""
    st = load().mv_codec_encode(_dev_ptr(idx), idx.stride(0), _dev_ptr(counts), counts_stride, n, idx.shape[0], d,
                                block_len, _dev_ptr(streams), streams.stride(0), _dev_ptr(n_bits),
                                _stream_handle(stream, idx))
    if st != MV_OK:
        raise MvError(st, "mv_codec_encode")


def mv_codec_decode(streams, n_bits, max_bits: int, d: int, block_len: int, idx_out, max_n: int, counts_out,
                    scratch, stream=None) -> None:
    st = load().mv_codec_decode(_dev_ptr(streams), streams.stride(0), _dev_ptr(n_bits), max_bits, streams.shape[0],
                                d, block_len, _dev_ptr(idx_out), idx_out.stride(0), max_n, _dev_ptr(counts_out),
                                _dev_ptr(scratch), scratch.numel() * scratch.element_size(), _stream_handle(stream, streams))
    if st != MV_OK:
        raise MvError(st, "mv_codec_decode")


MV_CODEC_STATIC_SCRATCH_BYTES = 16 << 20


def mv_codec_decode_static(streams, n_bits, max_bits: int, d: int, block_len: int, idx_out, max_n: int, counts_out,
                           stream=None) -> None:
    """mv_codec_decode on the library's own scratch array: allocates nothing."""
    st = load().mv_codec_decode_static(_dev_ptr(streams), streams.stride(0), _dev_ptr(n_bits), max_bits,
                                       streams.shape[0], d, block_len, _dev_ptr(idx_out), idx_out.stride(0), max_n,
                                       _dev_ptr(counts_out), _stream_handle(stream, streams))
    if st != MV_OK:
        raise MvError(st, "mv_codec_decode_static")


def mv_quant_scratch_bytes(n: int, rows: int, q: int) -> int:
    return int(load().mv_quant_scratch_bytes(n, rows, q))


def mv_quant_encode(vals, q: int, streams, means, scratch, stream=None) -> None:
    """vals: rows x n float32 device tensor; streams: rows x ld_words int32 (out);
    means: rows x 2**(q-1) float32 (out)."""
    st = load().mv_quant_encode(_dev_ptr(vals), vals.stride(0), vals.shape[1], vals.shape[0], q, _dev_ptr(streams),
                                streams.stride(0), _dev_ptr(means), _dev_ptr(scratch),
                                scratch.numel() * scratch.element_size(), _stream_handle(stream, vals))
    if st != MV_OK:
        raise MvError(st, "mv_quant_encode")


def mv_quant_decode(streams, n: int, q: int, means, out, stream=None) -> None:
    st = load().mv_quant_decode(_dev_ptr(streams), streams.stride(0), n, streams.shape[0], q, _dev_ptr(means),
                                _dev_ptr(out), out.stride(0), _stream_handle(stream, out))
    if st != MV_OK:
        raise MvError(st, "mv_quant_decode")


# ---- gradient norm over many tensors, and clipping ---------------------------------

_dtypes = None      # torch.float32 and torch.bfloat16 to mv_dtype, once torch is there
_int32 = None       # torch.int32, set with them


def _types():
    global _dtypes, _int32
    if _dtypes is None:
        import torch
        _int32 = torch.int32
        _dtypes = {torch.float32: MV_F32, torch.bfloat16: MV_BF16}
    return _dtypes


def _value_type(t, what: str) -> int:
    """mv_dtype of a float32 or bfloat16 tensor."""
    d = (_dtypes or _types()).get(t.dtype)
    if d is None:
        raise ValueError("%s is %s: float32 or bfloat16 is wanted" % (what, t.dtype))
    return d


def _float32(t, what: str, numel: int, device: int) -> int:
    """Address of a contiguous float32 device tensor of at least numel values; 0 for None."""
    if t is None:
        return 0
    if (_dtypes or _types()).get(t.dtype) != MV_F32 or not t.is_contiguous() or t.numel() < numel or t.get_device() != device:
        raise ValueError("%s has to be contiguous float32 of %d values or more on the same GPU" % (what, numel))
    return t.data_ptr()


def _pieces(t, o):
    """A tensor and where its clipped values go (or None) as pairs of contiguous pieces in the same order of elements."""
    if o is not None and o.shape != t.shape:
        raise ValueError("a tensor of shape %s does not go to one of %s" % (tuple(t.shape), tuple(o.shape)))
    if t.is_contiguous() and (o is None or o.is_contiguous()):
        yield t, o
        return
    # dense in another order of its dimensions, as both have it
    order = sorted(range(t.dim()), key=lambda i: -t.stride(i))
    p, q = t.permute(order), o.permute(order) if o is not None else None
    if p.is_contiguous() and (q is None or q.is_contiguous()):
        yield p, q
        return
    if t.dim() < 2:
        raise ValueError("a gradient's elements have to lie one behind the other in its last dimension")
    for i in range(t.shape[0]):
        yield from _pieces(t[i], o[i] if o is not None else None)


class _Clip(ctypes.c_void_p):
    """Handle of mv_clip_begin, with what the calls on it check against."""
    n_groups = 0
    device = -1
    groups = ()         # of each tensor given
    rows = None         # the list the library has
    writes = False


def _clip_list(tensors, out, groups, device):
    """The list as the library takes it: a numpy array of mv_clip_tensor."""
    import numpy as np
    out = list(out) if out is not None else None
    if not tensors or (out is not None and len(out) != len(tensors)):
        raise ValueError("as many tensors to write as to read, and at least one")
    if len(groups) != len(tensors):
        raise ValueError("a group for each tensor is wanted")
    both = tensors if out is None else tensors + out
    if any([t.get_device() != device for t in both]):
        raise ValueError("all tensors have to be on one GPU")
    if not all([t.is_contiguous() for t in both]):
        pieces = [(a, b, g) for i, g in enumerate(groups) for a, b in _pieces(tensors[i], out[i] if out is not None else None)]
        tensors, groups = [p[0] for p in pieces], [p[2] for p in pieces]
        out = [p[1] for p in pieces] if out is not None else None
    elif out is not None and [t.shape for t in tensors] != [t.shape for t in out]:
        raise ValueError("a tensor does not go to one of another shape")
    types = _types()
    rows = np.zeros(len(tensors), dtype=np.dtype(mv_clip_tensor))
    try:
        rows["src_dtype"] = [types[t.dtype] for t in tensors]
        if out is not None:
            rows["dst_dtype"] = [types[t.dtype] for t in out]
    except KeyError as e:
        raise ValueError("a gradient or its place is %s: float32 or bfloat16 is wanted" % e) from None
    rows["src"] = [t.data_ptr() for t in tensors]
    rows["numel"] = [t.numel() for t in tensors]
    rows["group"] = groups
    if out is not None:
        rows["dst"] = [t.data_ptr() for t in out]
    return rows


def mv_clip_begin(tensors, out=None, groups=None, norm: int = MV_NORM_L2, n_groups: Optional[int] = None,
                  workspace: int = 0, workspace_bytes: int = 0) -> _Clip:
    """A handle for the gradients `tensors` (torch device tensors, float32 or bfloat16, any mixture), groups[i] being the
    group that tensor i counts for (all one group by default).  out[i] is where its clipped values go: a tensor of the
    same shape, a view of a matrix row for instance, or tensors[i] itself; None: norms only.  Tensors that are not
    dense are taken apart into rows; both have to be dense in the same order.  Keep all of them alive and in place as
    long as the handle uses them (mv_clip_bind gives it others).  End it with mv_clip_end and mv_clip_release."""
    tensors = list(tensors)
    device = tensors[0].get_device() if tensors else -1
    groups = [0] * len(tensors) if groups is None else [int(g) for g in groups]
    rows = _clip_list(tensors, out, groups, device)
    n_groups = max(groups) + 1 if n_groups is None else int(n_groups)
    cfg = mv_clip_config(ctypes.sizeof(mv_clip_config), device, n_groups, norm, workspace or None, workspace_bytes)
    h = _Clip()
    st = load().mv_clip_begin(ctypes.byref(cfg), rows.ctypes.data, len(rows), ctypes.byref(h))
    if st != MV_OK:
        raise MvError(st, "mv_clip_begin")
    h.n_groups, h.device, h.groups, h.rows, h.writes = n_groups, device, groups, rows, out is not None
    return h


def mv_clip_bind(clip: _Clip, tensors, out=None, stream=None) -> None:
    """The handle's tensors from now on (in the stream's order): others of the same sizes, types and strides."""
    tensors = list(tensors)
    if (out is None) != (not clip.writes):
        raise ValueError("the handle was made %s places to write to" % ("with" if clip.writes else "without"))
    rows = _clip_list(tensors, out, clip.groups, clip.device)
    if len(rows) != len(clip.rows) or any((rows[f] != clip.rows[f]).any() for f in ("numel", "group", "src_dtype", "dst_dtype")):
        raise ValueError("the tensors' sizes, types and strides have to be those the handle was made for")
    pointers = rows["src"].copy(), rows["dst"].copy()
    st = load().mv_clip_bind(clip, pointers[0].ctypes.data, pointers[1].ctypes.data, _stream_handle(stream, tensors[0]))
    if st != MV_OK:
        raise MvError(st, "mv_clip_bind")


def mv_clip_norms(clip: _Clip, norms, stream=None) -> None:
    """norms: n_groups float32 on the device, out."""
    st = (_lib or load()).mv_clip_norms(clip, _float32(norms, "norms", clip.n_groups, clip.device), _stream_handle(stream, norms))
    if st != MV_OK:
        raise MvError(st, "mv_clip_norms")


def mv_clip_grads(clip: _Clip, max_norm: float, norms, coefs=None, stream=None) -> None:
    """The clipped gradients in the handle's `out` tensors; norms and coefs (may be None): n_groups float32, out."""
    st = (_lib or load()).mv_clip_grads(clip, max_norm, _float32(norms, "norms", clip.n_groups, clip.device),
                              _float32(coefs, "coefs", clip.n_groups, clip.device), _stream_handle(stream, norms))
    if st != MV_OK:
        raise MvError(st, "mv_clip_grads")


def mv_clip_set_spin_limit(clip: _Clip, polls: int) -> None:
    st = load().mv_clip_set_spin_limit(clip, polls)
    if st != MV_OK:
        raise MvError(st, "mv_clip_set_spin_limit")


def mv_clip_end(clip: _Clip) -> None:
    st = load().mv_clip_end(clip)
    if st != MV_OK:
        raise MvError(st, "mv_clip_end")


def mv_clip_release(clip: _Clip) -> None:
    """Frees the handle, which must not be used any more."""
    load().mv_clip_release(clip)
    clip.value = None


# ---- microscaled 4-bit floating point ----------------------------------------------


def mv_mx_row_words(n: int) -> int:
    return int(load().mv_mx_row_words(n))


def mv_mx_row_scales(n: int) -> int:
    return int(load().mv_mx_row_scales(n))


def _matrix(t, what: str, rows: int, n: int, device: int):
    """(address, mv_dtype, row stride) of a float32 or bfloat16 matrix with unit column stride."""
    d = (_dtypes or _types()).get(t.dtype)
    ld, step = t.stride()
    if d is None or step != 1 or t.get_device() != device or t.shape != (rows, n):
        d = _value_type(t, what)
        if t.shape != (rows, n) or t.get_device() != device:
            raise ValueError("%s is %s on GPU %d: %s on GPU %d is wanted" % (what, tuple(t.shape), t.get_device(), (rows, n), device))
        if n > 1:
            raise ValueError("%s has a column stride of %d: 1 is wanted" % (what, step))
    return t.data_ptr(), d, ld if rows > 1 else max(ld, n)


def _codes(codes, scales, rows: int, n: int, device: int, what: str = "codes"):
    """(address, row stride) of both, for `rows` rows of n values."""
    (r, words), (q, places) = codes.shape, scales.shape
    (ld_c, step_c), (ld_s, step_s) = codes.stride(), scales.stride()
    blocks = (n + 31) // 32
    if (r < rows or q < rows or words < 4 * blocks or places < (blocks + 3) // 4 * 4 or step_c != 1 or step_s != 1
            or codes.get_device() != device or scales.get_device() != device or codes.element_size() != 4
            or scales.element_size() != 1):
        raise ValueError("%s and scales have to be %d rows of mv_mx_row_words(%d) 32-bit words and mv_mx_row_scales(%d) bytes "
                         "or more, on the same GPU" % (what, rows, n, n))
    return codes.data_ptr(), ld_c, scales.data_ptr(), ld_s


def _scratch_of(scratch, device: int):
    if scratch is None:
        return 0, 0
    if scratch.get_device() != device or not scratch.is_contiguous():
        raise ValueError("scratch has to be contiguous memory on the same GPU")
    return scratch.data_ptr(), scratch.nbytes


def mv_mx_encode(vals, codes, scales, resid=None, stream=None) -> None:
    """vals: rows x n float32 or bfloat16; codes: rows x mv_mx_row_words(n) int32 (out); scales: rows x
    mv_mx_row_scales(n) uint8 (out); resid: rows x n float32 (out), vals less what the codes stand for; vals itself
    may be given."""
    rows, n = vals.shape
    device = vals.get_device()
    v, d, ld = _matrix(vals, "vals", rows, n, device)
    c, ld_c, s, ld_s = _codes(codes, scales, rows, n, device)
    r, ld_r = 0, 0
    if resid is not None:
        r, rd, ld_r = _matrix(resid, "resid", rows, n, device)
        if rd != MV_F32:
            raise ValueError("resid has to be float32")
    st = (_lib or load()).mv_mx_encode(v, d, ld, rows, n, c, ld_c, s, ld_s, r, ld_r, _stream_handle(stream, vals))
    if st != MV_OK:
        raise MvError(st, "mv_mx_encode")


def mv_mx_encode_t(vals, codes, scales, stream=None) -> None:
    """The columns of vals (rows x n): codes: n x mv_mx_row_words(rows), scales: n x mv_mx_row_scales(rows) (out)."""
    rows, n = vals.shape
    device = vals.get_device()
    v, d, ld = _matrix(vals, "vals", rows, n, device)
    st = (_lib or load()).mv_mx_encode_t(v, d, ld, rows, n, *_codes(codes, scales, n, rows, device), _stream_handle(stream, vals))
    if st != MV_OK:
        raise MvError(st, "mv_mx_encode_t")


def mv_mx_decode(codes, scales, out, stream=None) -> None:
    """out: rows x n float32 or bfloat16 (out), what the codes stand for."""
    rows, n = out.shape
    device = out.get_device()
    o, d, ld = _matrix(out, "out", rows, n, device)
    st = (_lib or load()).mv_mx_decode(*_codes(codes, scales, rows, n, device), rows, n, o, d, ld, _stream_handle(stream, out))
    if st != MV_OK:
        raise MvError(st, "mv_mx_decode")


def mv_mx_aggregate(codes, scales, weights, agg, stream=None) -> None:
    """agg: n float32 (out), the rows' weighted sum; weights: a float32 for each row of codes, or None for the mean."""
    rows, n, device = codes.shape[0], agg.numel(), agg.get_device()
    st = (_lib or load()).mv_mx_aggregate(*_codes(codes, scales, rows, n, device), rows, n, _float32(weights, "weights", rows, device),
                                _float32(agg, "agg", n, device), _stream_handle(stream, agg))
    if st != MV_OK:
        raise MvError(st, "mv_mx_aggregate")


def mv_mx_product_scratch_bytes(m: int, n: int, k: int) -> int:
    return (_lib or load()).mv_mx_product_scratch_bytes(m, n, k)


def mv_mx_product(a_codes, a_scales, b_codes, b_scales, k: int, out, scratch=None, stream=None) -> None:
    """out (m x n, float32 or bfloat16) = a b^T: a of m rows and b of n rows, k values each, in 4 bits along k.
    scratch: mv_mx_product_scratch_bytes(m, n, k) bytes."""
    m, n = out.shape
    device = out.get_device()
    o, d, ld = _matrix(out, "out", m, n, device)
    st = (_lib or load()).mv_mx_product(*_codes(a_codes, a_scales, m, k, device, "a_codes"), *_codes(b_codes, b_scales, n, k, device, "b_codes"),
                              m, n, k, o, d, ld, *_scratch_of(scratch, device), _stream_handle(stream, out))
    if st != MV_OK:
        raise MvError(st, "mv_mx_product")


def mv_mx_linear_scratch_bytes(m: int, n: int, k: int) -> int:
    return (_lib or load()).mv_mx_linear_scratch_bytes(m, n, k)


def mv_mx_linear(x, w_codes, w_scales, out, scratch, stream=None) -> None:
    """out (m x n) = q(x) w^T: x m x k, rounded to 4 bits as mv_mx_encode does; w: n rows of k values in 4 bits."""
    m, k = x.shape
    n = out.shape[1]
    device = out.get_device()
    a, xd, ld_x = _matrix(x, "x", m, k, device)
    o, d, ld = _matrix(out, "out", m, n, device)
    st = (_lib or load()).mv_mx_linear(a, xd, ld_x, *_codes(w_codes, w_scales, n, k, device, "w_codes"), m, n, k, o, d, ld,
                             *_scratch_of(scratch, device), _stream_handle(stream, out))
    if st != MV_OK:
        raise MvError(st, "mv_mx_linear")


def mv_mx_linear_grad_scratch_bytes(m: int, n: int, k: int) -> int:
    return (_lib or load()).mv_mx_linear_grad_scratch_bytes(m, n, k)


def mv_mx_linear_grad(x, dy, wt_codes, wt_scales, dx, dw, scratch, stream=None) -> None:
    """dx (m x k) = q(dy) wt^T and dw (n x k) = qt(dy) qt(x)^T of mv_mx_linear's product; wt: the weights' columns, k
    rows of n values in 4 bits.  dx (with wt_codes and wt_scales) or dw (with x) may be None; x and dy have one type."""
    m, n = dy.shape
    device = dy.get_device()
    k = dx.shape[1] if dx is not None else x.shape[1]
    g, yd, ld_dy = _matrix(dy, "dy", m, n, device)
    a, ld_x, w, o, od, ld_dx, p, pd, ld_dw = 0, 0, (0, 0, 0, 0), 0, 0, 0, 0, 0, 0
    if dx is not None:
        w = _codes(wt_codes, wt_scales, k, n, device, "wt_codes")
        o, od, ld_dx = _matrix(dx, "dx", m, k, device)
    if dw is not None:
        a, xd, ld_x = _matrix(x, "x", m, k, device)
        if xd != yd:
            raise ValueError("x and dy have to be of one type")
        p, pd, ld_dw = _matrix(dw, "dw", n, k, device)
    st = (_lib or load()).mv_mx_linear_grad(a, ld_x, g, ld_dy, yd, *w, m, n, k, o, od, ld_dx, p, pd, ld_dw,
                                  *_scratch_of(scratch, device), _stream_handle(stream, dy))
    if st != MV_OK:
        raise MvError(st, "mv_mx_linear_grad")


# ---- 8-bit floating point by blocks of 128 ----------------------------------


def mv_f8_row_bytes(n: int) -> int:
    return int(load().mv_f8_row_bytes(n))


def mv_f8_row_scales(n: int) -> int:
    return int(load().mv_f8_row_scales(n))


def _bytes(codes, scales, rows: int, n: int, device: int, what: str = "codes"):
    """(address, row stride) of 8-bit codes and their scales, for `rows` rows of n values."""
    (r, length), (q, places) = codes.shape, scales.shape
    (ld_c, step_c), (ld_s, step_s) = codes.stride(), scales.stride()
    blocks = (n + 127) // 128
    if (r < rows or q < rows or length < 128 * blocks or places < (blocks + 3) // 4 * 4 or step_c != 1 or step_s != 1
            or codes.get_device() != device or scales.get_device() != device or codes.element_size() != 1
            or scales.element_size() != 1):
        raise ValueError("%s and scales have to be %d rows of mv_f8_row_bytes(%d) and mv_f8_row_scales(%d) bytes or more, on the "
                         "same GPU" % (what, rows, n, n))
    return codes.data_ptr(), ld_c, scales.data_ptr(), ld_s


def mv_f8_encode(vals, codes, scales, stream=None) -> None:
    """vals: rows x n float32 or bfloat16; codes: rows x mv_f8_row_bytes(n) uint8 (out); scales: rows x
    mv_f8_row_scales(n) uint8 (out)."""
    rows, n = vals.shape
    device = vals.get_device()
    v, d, ld = _matrix(vals, "vals", rows, n, device)
    st = (_lib or load()).mv_f8_encode(v, d, ld, rows, n, *_bytes(codes, scales, rows, n, device), _stream_handle(stream, vals))
    if st != MV_OK:
        raise MvError(st, "mv_f8_encode")


def mv_f8_encode_t(vals, codes, scales, stream=None) -> None:
    """The columns of vals (rows x n): codes: n x mv_f8_row_bytes(rows), scales: n x mv_f8_row_scales(rows) (out)."""
    rows, n = vals.shape
    device = vals.get_device()
    v, d, ld = _matrix(vals, "vals", rows, n, device)
    st = (_lib or load()).mv_f8_encode_t(v, d, ld, rows, n, *_bytes(codes, scales, n, rows, device), _stream_handle(stream, vals))
    if st != MV_OK:
        raise MvError(st, "mv_f8_encode_t")


def mv_f8_decode(codes, scales, out, stream=None) -> None:
    """out: rows x n float32 or bfloat16 (out), what the codes stand for."""
    rows, n = out.shape
    device = out.get_device()
    o, d, ld = _matrix(out, "out", rows, n, device)
    st = (_lib or load()).mv_f8_decode(*_bytes(codes, scales, rows, n, device), rows, n, o, d, ld, _stream_handle(stream, out))
    if st != MV_OK:
        raise MvError(st, "mv_f8_decode")


def mv_f8_product_scratch_bytes(m: int, n: int, k: int) -> int:
    return (_lib or load()).mv_f8_product_scratch_bytes(m, n, k)


def mv_f8_product(a_codes, a_scales, b_codes, b_scales, k: int, out, scratch=None, stream=None) -> None:
    """out (m x n, float32 or bfloat16) = a b^T: a of m rows and b of n rows, k values each, in 8 bits along k.
    scratch: mv_f8_product_scratch_bytes(m, n, k) bytes."""
    m, n = out.shape
    device = out.get_device()
    o, d, ld = _matrix(out, "out", m, n, device)
    st = (_lib or load()).mv_f8_product(*_bytes(a_codes, a_scales, m, k, device, "a_codes"), *_bytes(b_codes, b_scales, n, k, device, "b_codes"),
                              m, n, k, o, d, ld, *_scratch_of(scratch, device), _stream_handle(stream, out))
    if st != MV_OK:
        raise MvError(st, "mv_f8_product")


def mv_f8_linear_scratch_bytes(m: int, n: int, k: int) -> int:
    return (_lib or load()).mv_f8_linear_scratch_bytes(m, n, k)


def mv_f8_linear(x, w_codes, w_scales, out, scratch, stream=None) -> None:
    """out (m x n) = q(x) w^T: x m x k, rounded to 8 bits as mv_f8_encode does; w: n rows of k values in 8 bits."""
    m, k = x.shape
    n = out.shape[1]
    device = out.get_device()
    a, xd, ld_x = _matrix(x, "x", m, k, device)
    o, d, ld = _matrix(out, "out", m, n, device)
    st = (_lib or load()).mv_f8_linear(a, xd, ld_x, *_bytes(w_codes, w_scales, n, k, device, "w_codes"), m, n, k, o, d, ld,
                             *_scratch_of(scratch, device), _stream_handle(stream, out))
    if st != MV_OK:
        raise MvError(st, "mv_f8_linear")


def mv_f8_linear_grad_scratch_bytes(m: int, n: int, k: int) -> int:
    return (_lib or load()).mv_f8_linear_grad_scratch_bytes(m, n, k)


def mv_f8_linear_grad(x, dy, wt_codes, wt_scales, dx, dw, scratch, stream=None) -> None:
    """dx (m x k) = q(dy) wt^T and dw (n x k) = qt(dy) qt(x)^T of mv_f8_linear's product; wt: the weights' columns, k
    rows of n values in 8 bits.  dx (with wt_codes and wt_scales) or dw (with x) may be None; x and dy have one type."""
    m, n = dy.shape
    device = dy.get_device()
    k = dx.shape[1] if dx is not None else x.shape[1]
    g, yd, ld_dy = _matrix(dy, "dy", m, n, device)
    a, ld_x, w, o, od, ld_dx, p, pd, ld_dw = 0, 0, (0, 0, 0, 0), 0, 0, 0, 0, 0, 0
    if dx is not None:
        w = _bytes(wt_codes, wt_scales, k, n, device, "wt_codes")
        o, od, ld_dx = _matrix(dx, "dx", m, k, device)
    if dw is not None:
        a, xd, ld_x = _matrix(x, "x", m, k, device)
        if xd != yd:
            raise ValueError("x and dy have to be of one type")
        p, pd, ld_dw = _matrix(dw, "dw", n, k, device)
    st = (_lib or load()).mv_f8_linear_grad(a, ld_x, g, ld_dy, yd, *w, m, n, k, o, od, ld_dx, p, pd, ld_dw,
                                  *_scratch_of(scratch, device), _stream_handle(stream, dy))
    if st != MV_OK:
        raise MvError(st, "mv_f8_linear_grad")


# ---- layer norm ---------------------------------------------------------------


def _weights(a, b, n: int, device: int):
    """(address of gamma, address of beta, mv_dtype) of float32 or bfloat16 vectors of one type, either may be None."""
    kinds, d, at = _dtypes or _types(), None, [0, 0]
    for i, t in enumerate((a, b)):
        if t is not None:
            kind = kinds.get(t.dtype)
            if kind is None or t.numel() != n or not t.is_contiguous() or t.get_device() != device or (d is not None and kind != d):
                raise ValueError("%s has to be %d contiguous float32 or bfloat16 values on the same GPU, of the other weights' type"
                                 % (("gamma", "beta")[i], n))
            d = kind
            at[i] = t.data_ptr()
    return at[0], at[1], MV_F32 if d is None else d


def mv_layernorm_forward(x, gamma, beta, eps: float, out, mean=None, rstd=None, stream=None) -> None:
    """out (rows x n, float32 or bfloat16; may be x) = the layer norm of x's rows; gamma, beta: n float32 or bfloat16 values
    or None; mean, rstd: rows float32 (out) or None, for mv_layernorm_backward."""
    rows, n = x.shape
    device = x.get_device()
    a, xd, ld_x = _matrix(x, "x", rows, n, device)
    o, od, ld_o = _matrix(out, "out", rows, n, device)
    g, b, wd = _weights(gamma, beta, n, device)
    st = (_lib or load()).mv_layernorm_forward(a, xd, ld_x, rows, n, g, b, wd, eps, o, od, ld_o, _float32(mean, "mean", rows, device),
                                               _float32(rstd, "rstd", rows, device), _stream_handle(stream, x))
    if st != MV_OK:
        raise MvError(st, "mv_layernorm_forward")


def mv_layernorm_scratch_bytes(rows: int, n: int) -> int:
    return (_lib or load()).mv_layernorm_scratch_bytes(rows, n)


def mv_layernorm_backward(x, dy, gamma, mean, rstd, dx, dgamma, dbeta, scratch, stream=None) -> None:
    """The gradients of mv_layernorm_forward's x (dx: rows x n, may be dy or x), gamma and beta (n float32 each) from dy; each
    may be None.  x and dy have one type; scratch: mv_layernorm_scratch_bytes(rows, n) bytes."""
    rows, n = x.shape
    device = x.get_device()
    a, xd, ld_x = _matrix(x, "x", rows, n, device)
    g, yd, ld_dy = _matrix(dy, "dy", rows, n, device)
    if xd != yd:
        raise ValueError("x and dy have to be of one type")
    o, od, ld_o = _matrix(dx, "dx", rows, n, device) if dx is not None else (0, 0, 0)
    w, _, wd = _weights(gamma, None, n, device)
    st = (_lib or load()).mv_layernorm_backward(a, ld_x, g, ld_dy, xd, rows, n, w, wd, _float32(mean, "mean", rows, device),
                                                _float32(rstd, "rstd", rows, device), o, od, ld_o, _float32(dgamma, "dgamma", n, device),
                                                _float32(dbeta, "dbeta", n, device), *_scratch_of(scratch, device),
                                                _stream_handle(stream, x))
    if st != MV_OK:
        raise MvError(st, "mv_layernorm_backward")


# ---- distillation from a teacher's top logits ---------------------------------


def _list(idx, top, labels, rows: int, device: int):
    """(address and row stride of the coordinates; address, mv_dtype and row stride of the teacher's logits; entries of a row;
    address of the labels)."""
    i, ld_i, t, td, ld_t, k, at = 0, 0, 0, 0, 0, 0, 0
    if idx is not None:
        r, k = idx.shape
        ld_i, step = idx.stride()
        if r != rows or idx.dtype != _int32 or (k > 1 and step != 1) or idx.get_device() != device:
            raise ValueError("idx has to be %d rows of int32 on the same GPU, each in one piece" % rows)
        if k:
            if top is None:
                raise ValueError("idx names coordinates that top has no logits of")
            i, ld_i = idx.data_ptr(), ld_i if rows > 1 else max(ld_i, k)
            t, td, ld_t = _matrix(top, "top", rows, k, device)
    elif top is not None:
        raise ValueError("top has logits of coordinates that no idx names")
    if labels is not None:
        if labels.dtype != _int32 or labels.numel() != rows or not labels.is_contiguous() or labels.get_device() != device:
            raise ValueError("labels have to be %d contiguous int32 on the same GPU" % rows)
        at = labels.data_ptr()
    return i, ld_i, t, td, ld_t, k, at


def mv_distill_scratch_bytes(rows: int, n: int) -> int:
    return (_lib or load()).mv_distill_scratch_bytes(rows, n)


def mv_distill_loss(logits, idx, top, labels, temperature: float, soft: float, hard: float, loss, scratch=None, stats=None, dz=None,
                    grad=None, stream=None) -> None:
    """loss: rows float32 (out; may be None where dz is wanted); logits: rows x n float32 or bfloat16; idx, top: the teacher's
    coordinates (rows x k int32, any other than 0 .. n-1 is no entry) and logits (rows x k float32 or bfloat16), or both None;
    labels: rows int32 or None; stats: rows x 3 float32 (out) or None, for mv_distill_grad; dz: rows x n (out; may be logits)
    or None, with grad, rows float32, the gradients that arrive at the losses, None for 1."""
    rows, n = logits.shape
    device = logits.get_device()
    z, zd, ld_z = _matrix(logits, "logits", rows, n, device)
    o, od, ld_o = _matrix(dz, "dz", rows, n, device) if dz is not None else (0, 0, 0)
    c, size = _scratch_of(scratch, device)
    st = (_lib or load()).mv_distill_loss(z, zd, ld_z, rows, n, *_list(idx, top, labels, rows, device), temperature, soft, hard,
                                          _float32(loss, "loss", rows, device), _float32(stats, "stats", 3 * rows, device),
                                          _float32(grad, "grad", rows, device), o, od, ld_o, c, size, _stream_handle(stream, logits))
    if st != MV_OK:
        raise MvError(st, "mv_distill_loss")


def mv_distill_grad(logits, idx, top, labels, temperature: float, soft: float, hard: float, stats, dz, grad=None, stream=None) -> None:
    """dz of mv_distill_loss from the stats of a call with the same arguments."""
    rows, n = logits.shape
    device = logits.get_device()
    z, zd, ld_z = _matrix(logits, "logits", rows, n, device)
    o, od, ld_o = _matrix(dz, "dz", rows, n, device)
    st = (_lib or load()).mv_distill_grad(z, zd, ld_z, rows, n, *_list(idx, top, labels, rows, device), temperature, soft, hard,
                                          _float32(stats, "stats", 3 * rows, device), _float32(grad, "grad", rows, device), o, od, ld_o,
                                          _stream_handle(stream, logits))
    if st != MV_OK:
        raise MvError(st, "mv_distill_grad")

"""Thin ctypes binding of liblc.so: argument marshalling only, same names as include/lc.h and include/lc_serve.h.

Device buffers are torch CUDA tensors (torch is used for device memory and streams,
nothing else).  There is no CPU fallback: if the library is missing, importing fails.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_PATH = os.path.join(_HERE, "liblc.so")
if not os.path.exists(_PATH):
    raise ImportError("liblc.so is not built: run `python -m paper_2009_13003_amd.build` "
                      "(or __graft_entry__.build()) first")
_lib = ctypes.CDLL(_PATH)

OK, ERR_BADARG, ERR_NONFINITE, ERR_OUT_TOO_SMALL, ERR_BAD_BLOB, ERR_HIP, ERR_WORKSPACE = range(7)
MAX_N = 1 << 32
MAX_TICKETS = 32
MAX_MANY = 64
CHUNK = 16384

_u64, _i64, _int, _vp, _sz = ctypes.c_uint64, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
_lib.lc_encode_bound.restype = _sz
_lib.lc_encode_bound.argtypes = [_u64, _int]
_lib.lc_workspace_bytes.restype = _sz
_lib.lc_workspace_bytes.argtypes = [_u64, _int]
_lib.lc_set_workspace.restype = _int
_lib.lc_set_workspace.argtypes = [_vp, _sz]
_lib.lc_encode.restype = _i64
_lib.lc_encode.argtypes = [_vp, _vp, _u64, _int, _vp, _vp]
_lib.lc_set_option.restype = _int
_lib.lc_set_option.argtypes = [_int, _int]
_lib.lc_encode_sized.restype = _i64
_lib.lc_encode_sized.argtypes = [_vp, _vp, _u64, _int, _vp, _sz, _int, _vp]
_lib.lc_decode_sized.restype = _i64
_lib.lc_decode_sized.argtypes = [_vp, _sz, _vp, _u64, _int, _vp]
_lib.lc_verify.restype = _i64
_lib.lc_verify.argtypes = [_vp, _sz, _u64, _int, _vp]
_lib.lc_encode_static.restype = _int
_lib.lc_encode_static.argtypes = [_vp, _vp, _u64, _int, _vp, _vp]
_lib.lc_encode_t.restype = _i64
_lib.lc_encode_t.argtypes = [_vp, _vp, _u64, _int, _vp, _int, _vp]
_lib.lc_decode_t.restype = _i64
_lib.lc_decode_t.argtypes = [_vp, _vp, _u64, _int, _vp]
_lib.lc_batch_workspace_bytes.restype = _sz
_lib.lc_batch_workspace_bytes.argtypes = [ctypes.POINTER(_u64), _int, _int]
_lib.lc_encode_batch.restype = _i64
_lib.lc_encode_batch.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_u64), _int, _int,
                                 ctypes.POINTER(_vp), ctypes.POINTER(_i64), _vp]
_lib.lc_encode_batch_t.restype = _i64
_lib.lc_encode_batch_t.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_u64), _int, _int,
                                   ctypes.POINTER(_vp), ctypes.POINTER(_i64), _int, _vp]
_lib.lc_decode_batch_t.restype = _i64
_lib.lc_decode_batch_t.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_u64), _int, ctypes.POINTER(_i64), _int, _vp]
_lib.lc_decode_batch.restype = _i64
_lib.lc_decode_batch.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_u64), _int, ctypes.POINTER(_i64), _vp]
_lib.lc_encode_cached.restype = _i64
_lib.lc_encode_cached.argtypes = [_vp, _vp, _u64, _int, _vp, _vp, ctypes.POINTER(_int), _vp]
_lib.lc_encode_cached_t.restype = _i64
_lib.lc_encode_cached_t.argtypes = [_vp, _vp, _u64, _int, _vp, _int, _vp, ctypes.POINTER(_int), _vp]
_lib.lc_encode_async_t.restype = _int
_lib.lc_encode_async_t.argtypes = [_vp, _vp, _u64, _int, _vp, _int, _vp, _vp]
_lib.lc_encode_async.restype = _int
_lib.lc_encode_async.argtypes = [_vp, _vp, _u64, _int, _vp, _vp, _vp]
_lib.lc_encode_release_inputs.restype = _int
_lib.lc_encode_release_inputs.argtypes = [_int, _vp]
_lib.lc_encode_wait.restype = _i64
_lib.lc_encode_wait.argtypes = [_int, ctypes.POINTER(_int)]
_lib.lc_decode.restype = _i64
_lib.lc_decode.argtypes = [_vp, _vp, _u64, _vp]
_lib.lc_decode_many.restype = _i64
_lib.lc_decode_many_t.restype = _i64
_lib.lc_decode_many_t.argtypes = [ctypes.POINTER(_vp), _int, _vp, _u64, _int, _vp]
_lib.lc_decode_many.argtypes = [ctypes.POINTER(_vp), _int, _vp, _u64, _vp]
_lib.lc_blob_info.restype = _int
_lib.lc_blob_info.argtypes = [_vp, ctypes.POINTER(_u64), ctypes.POINTER(_int), ctypes.POINTER(_u64), ctypes.POINTER(_int)]
_lib.lc_blob_sizes.restype = _int
_lib.lc_blob_sizes.argtypes = [_vp, ctypes.POINTER(_u64)]
_lib.lc_shutdown.restype = None
_lib.lc_shutdown.argtypes = []
_lib.lc_strerror.restype = ctypes.c_char_p
_lib.lc_strerror.argtypes = [_int]
_lib.lc_profile.restype = _int
_lib.lc_profile.argtypes = [_int]
_lib.lc_profile_read.restype = _int
_lib.lc_profile_read.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_u64), _int]
_lib.lc_profile_name.restype = ctypes.c_char_p
_lib.lc_profile_name.argtypes = [_int]


class _W4(ctypes.Structure):            # struct lc_w4
    _fields_ = [("codes", _vp), ("scales", _vp), ("n", _u64), ("k", _u64), ("codes_pitch", _u64), ("scales_pitch", _u64), ("group", _int)]


class _I8(ctypes.Structure):            # struct lc_i8
    _fields_ = [("codes", _vp), ("scales", _vp), ("n", _u64), ("k", _u64), ("pitch", _u64)]


class _KvPages(ctypes.Structure):       # struct lc_kv_pages
    _fields_ = [("table", _vp), ("lens", _vp), ("free_pages", _vp), ("free_count", _vp), ("batch", _u64), ("ld_table", _u64), ("table_pages", _u64),
                ("free_room", _u64), ("page_tokens", _int)]


class _KvCache(ctypes.Structure):       # struct lc_kv_cache
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("pages", _u64), ("page_tokens", _int), ("heads", _int),
                ("dim", _int), ("bits", _int)]


_lib.lc_w4_row_bytes.restype = _sz
_lib.lc_w4_row_bytes.argtypes = [_u64]
_lib.lc_w4_quantize.restype = _int
_lib.lc_w4_quantize.argtypes = [_vp, _u64, _int, _vp, _vp]
_lib.lc_w4_dequantize.restype = _int
_lib.lc_w4_dequantize.argtypes = [_vp, _vp, _u64, _int, _vp]
_lib.lc_w4_matmul.restype = _int
_lib.lc_w4_matmul.argtypes = [_vp, _u64, _u64, _vp, _vp, _vp, _u64, _int, _vp]

_lib.lc_kv_write.restype = _int
_lib.lc_kv_write.argtypes = [_vp, _vp, _vp, _u64, _u64, _vp, _u64, _int, _vp]
_lib.lc_kv_read.restype = _int
_lib.lc_kv_read.argtypes = [_vp, _vp, _u64, _vp, _vp, _u64, _u64, _int, _vp]
_lib.lc_kv_workspace_bytes.restype = _sz
_lib.lc_kv_workspace_bytes.argtypes = [_u64, _int, _int, _int, _int]
_lib.lc_i8_quantize.restype = _int
_lib.lc_i8_quantize.argtypes = [_vp, _u64, _int, _vp, _vp]
_lib.lc_i8_dequantize.restype = _int
_lib.lc_i8_dequantize.argtypes = [_vp, _vp, _u64, _int, _vp]
_lib.lc_i8_matmul.restype = _int
_lib.lc_i8_matmul.argtypes = [_vp, _vp, _vp, _vp, _u64, _int, _vp]
_lib.lc_i8_workspace_bytes.restype = _sz
_lib.lc_i8_workspace_bytes.argtypes = [_u64, _u64]
_lib.lc_i8_linear.restype = _int
_lib.lc_i8_linear.argtypes = [_vp, _u64, _u64, _vp, _vp, _vp, _u64, _int, _vp, _sz, _vp]
_lib.lc_kv_prompt_workspace_bytes.restype = _sz
_lib.lc_kv_prompt_workspace_bytes.argtypes = [_u64, _u64, _int, _int, _int]
_lib.lc_kv_prompt_workspace_most.restype = _sz
_lib.lc_kv_prompt_workspace_most.argtypes = [_u64, _u64, _int, _int, _int]
_lib.lc_kv_attend_prompt.restype = _int
_lib.lc_kv_attend_prompt.argtypes = [_vp, _vp, _u64, _u64, _int, _vp, _u64, _vp, _u64, _u64, _vp, ctypes.c_float, _vp, _u64, _int, _vp, _sz, _vp]
_lib.lc_kv_extend.restype = _int
_lib.lc_kv_extend.argtypes = [_vp, _vp, _u64, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.lc_kv_trim.restype = _int
_lib.lc_kv_trim.argtypes = [_vp, _vp, _vp, _vp, _vp]
_lib.lc_draft_workspace_bytes.restype = _sz
_lib.lc_draft_workspace_bytes.argtypes = [_u64]
_lib.lc_draft_verify.restype = _int
_lib.lc_draft_verify.argtypes = [_vp, _u64, _u64, _u64, _int, _u64, _vp, _vp, _u64, _u64, _vp, _vp, _vp, _int, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.lc_kv_attend.restype = _int
_lib.lc_kv_attend.argtypes = [_vp, _vp, _u64, _int, _int, _vp, _u64, _u64, _vp, _vp, ctypes.c_float, _vp, _int, _vp, _sz, _vp]


class LcError(RuntimeError):
    def __init__(self, status):
        super().__init__("lc status %d: %s" % (status, lc_strerror(status)))
        self.status = status


def lc_strerror(status):
    return _lib.lc_strerror(int(status)).decode()


def lc_encode_bound(n, nbits):
    return int(_lib.lc_encode_bound(n, nbits))


def lc_workspace_bytes(n, nbits):
    return int(_lib.lc_workspace_bytes(n, nbits))


try:                                    # torch's current stream as a raw handle, without building a Stream object
    _raw_current_stream = torch._C._cuda_getCurrentRawStream
    _current_device = torch._C._cuda_getDevice
except AttributeError:                  # (other torch builds: the public, slower way)
    _raw_current_stream = None


def _stream(stream):
    if stream is None:
        if _raw_current_stream is not None:
            return ctypes.c_void_p(_raw_current_stream(_current_device()))
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _dev_f32(t):
    assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous(), "need a contiguous CUDA float32 tensor"
    return ctypes.c_void_p(t.data_ptr())


def lc_set_workspace(ws):
    """ws: a CUDA uint8 tensor (kept alive by the caller) or None."""
    if ws is None:
        return int(_lib.lc_set_workspace(None, 0))
    assert ws.is_cuda and ws.dtype == torch.uint8 and ws.is_contiguous()
    return int(_lib.lc_set_workspace(ctypes.c_void_p(ws.data_ptr()), ws.numel()))


def lc_encode(w, w_ref, nbits, out, stream=None, n=None):
    """Returns the blob size in bytes (blob is out[:size]); raises LcError on a negative status."""
    n = w.numel() if n is None else n
    assert out.is_cuda and out.dtype == torch.uint8 and out.is_contiguous()
    assert out.numel() >= lc_encode_bound(n, nbits) > 0 or not (1 <= nbits <= 4), "out is smaller than lc_encode_bound"
    r = int(_lib.lc_encode(_dev_f32(w), _dev_f32(w_ref), n, nbits, ctypes.c_void_p(out.data_ptr()), _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r


STATIC_MAX_N = 1 << 23


def lc_encode_static(w, w_ref, nbits, out, stream=None, n=None):
    """lc_encode without any allocation and without waiting: enqueues only; the blob's size and status are in its
    header once the stream has run the call.  Raises LcError on a status other than LC_OK."""
    n = w.numel() if n is None else n
    assert out.is_cuda and out.dtype == torch.uint8 and out.is_contiguous()
    assert out.numel() >= lc_encode_bound(n, nbits) > 0 or not (1 <= nbits <= 4), "out is smaller than lc_encode_bound"
    st = int(_lib.lc_encode_static(_dev_f32(w), _dev_f32(w_ref), n, nbits, ctypes.c_void_p(out.data_ptr()), _stream(stream)))
    if st != OK:
        raise LcError(st)


DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, torch.float64: 3}


def _dev_any(t):
    assert t.is_cuda and t.dtype in DTYPES and t.is_contiguous(), "need a contiguous CUDA float32 / bfloat16 / float16 / float64 tensor"
    return ctypes.c_void_p(t.data_ptr())


def lc_encode_t(w, w_ref, nbits, out, stream=None, n=None):
    """lc_encode for float32, bfloat16, float16 or float64 parameters (w and w_ref of the same dtype)."""
    n = w.numel() if n is None else n
    assert w.dtype == w_ref.dtype
    assert out.is_cuda and out.dtype == torch.uint8 and out.is_contiguous()
    assert out.numel() >= lc_encode_bound(n, nbits) > 0 or not (1 <= nbits <= 4), "out is smaller than lc_encode_bound"
    r = int(_lib.lc_encode_t(_dev_any(w), _dev_any(w_ref), n, nbits, ctypes.c_void_p(out.data_ptr()), DTYPES[w.dtype], _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r


def lc_decode_t(blob, w_ref, stream=None, n=None):
    """lc_decode for float32, bfloat16, float16 or float64 parameters."""
    n = w_ref.numel() if n is None else n
    assert blob.is_cuda and blob.dtype == torch.uint8 and blob.is_contiguous()
    r = int(_lib.lc_decode_t(ctypes.c_void_p(blob.data_ptr()), _dev_any(w_ref), n, DTYPES[w_ref.dtype], _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r


OPT_KEY_STAGING, STAGING_AUTO, STAGING_ALWAYS, STAGING_NEVER = 1, 0, 1, 2
OPT_VERIFY_FIRST = 2


def lc_set_option(option, value):
    st = int(_lib.lc_set_option(option, value))
    if st != OK:
        raise LcError(st)


def lc_encode_sized(w, w_ref, nbits, out, stream=None, n=None):
    """lc_encode_t with the size of `out` stated: ERR_OUT_TOO_SMALL if it is below lc_encode_bound."""
    n = w.numel() if n is None else n
    assert w.dtype == w_ref.dtype and out.is_cuda and out.dtype == torch.uint8 and out.is_contiguous()
    r = int(_lib.lc_encode_sized(_dev_any(w), _dev_any(w_ref), n, nbits, ctypes.c_void_p(out.data_ptr()), out.numel(),
                                 DTYPES[w.dtype], _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r


def lc_decode_sized(blob, w_ref, stream=None, n=None):
    """lc_decode_t with the size of `blob` stated: a header that claims more bytes is refused."""
    n = w_ref.numel() if n is None else n
    assert blob.is_cuda and blob.dtype == torch.uint8 and blob.is_contiguous()
    r = int(_lib.lc_decode_sized(ctypes.c_void_p(blob.data_ptr()), blob.numel(), _dev_any(w_ref), n, DTYPES[w_ref.dtype],
                                 _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r


class EncodeBatch:
    """The marshalled arguments of one lc_encode_batch call, kept for the next call on the same tensors: a
    training loop checkpoints the same parameter tensors every time, and checking and converting a few hundred
    tensors costs more host time than the call.  The tensors must stay alive and in place."""

    def __init__(self, ws, w_refs, nbits, outs):
        count = len(ws)
        assert count == len(w_refs) == len(outs) and count >= 1
        self.dtype = ws[0].dtype                             # float32, bfloat16 or float16, the same for every tensor
        for w, r, o in zip(ws, w_refs, outs):
            assert w.is_cuda and w.dtype == self.dtype and w.is_contiguous() and r.is_cuda and r.dtype == self.dtype
            assert r.is_contiguous() and r.numel() == w.numel() and o.is_cuda and o.dtype == torch.uint8 and o.is_contiguous()
            assert o.numel() >= lc_encode_bound(w.numel(), nbits) > 0 or not (1 <= nbits <= 4), "out is smaller than lc_encode_bound"
        self.keep = (list(ws), list(w_refs), list(outs))
        self.count, self.nbits = count, nbits
        self.wp = (_vp * count)(*[t.data_ptr() if t.numel() else None for t in ws])
        self.rp = (_vp * count)(*[t.data_ptr() if t.numel() else None for t in w_refs])
        self.op = (_vp * count)(*[t.data_ptr() for t in outs])
        self.ns = (_u64 * count)(*[t.numel() for t in ws])
        self.sizes = (_i64 * count)()

    def run(self, stream=None):
        if self.dtype == torch.float32:
            r = int(_lib.lc_encode_batch(self.wp, self.rp, self.ns, self.count, self.nbits, self.op, self.sizes, _stream(stream)))
        else:
            r = int(_lib.lc_encode_batch_t(self.wp, self.rp, self.ns, self.count, self.nbits, self.op, self.sizes,
                                           DTYPES[self.dtype], _stream(stream)))
        sizes = list(self.sizes)
        if r < 0 and all(s >= 0 for s in sizes):
            raise LcError(-r)
        return sizes


def lc_encode_batch(ws, w_refs, nbits, outs, stream=None):
    """One table per tensor, all tensors in one call. Returns the list of blob sizes (negative: -(status) of that
    tensor); raises LcError only for errors that concern the whole call."""
    return EncodeBatch(ws, w_refs, nbits, outs).run(stream)


lc_encode_batch_t = lc_encode_batch      # (EncodeBatch picks the entry point by the tensors' dtype)


def lc_blob_sizes(header_bytes):
    """Checkpoint size in bits after each stage (Section 4.3): dict(E, EP, EPH), from the first 64+ bytes of a blob."""
    buf = ctypes.create_string_buffer(bytes(header_bytes[:512]), 512)
    bits = (_u64 * 3)()
    st = int(_lib.lc_blob_sizes(buf, bits))
    if st != 0:
        raise LcError(st)
    return dict(E=int(bits[0]), EP=int(bits[1]), EPH=int(bits[2]))


class DecodeBatch:
    """The marshalled arguments of one lc_decode_batch call, kept for the next call on the same tensors (see EncodeBatch)."""

    def __init__(self, blobs, w_refs):
        count = len(blobs)
        assert count == len(w_refs) and count >= 1
        self.dtype = w_refs[0].dtype
        for b, r in zip(blobs, w_refs):
            assert b.is_cuda and b.dtype == torch.uint8 and b.is_contiguous()
            assert r.is_cuda and r.dtype == self.dtype and r.is_contiguous()
        self.keep = (list(blobs), list(w_refs))
        self.count = count
        self.bp = (_vp * count)(*[t.data_ptr() for t in blobs])
        self.rp = (_vp * count)(*[t.data_ptr() if t.numel() else None for t in w_refs])
        self.ns = (_u64 * count)(*[t.numel() for t in w_refs])
        self.sizes = (_i64 * count)()

    def run(self, stream=None):
        if self.dtype == torch.float32:
            r = int(_lib.lc_decode_batch(self.bp, self.rp, self.ns, self.count, self.sizes, _stream(stream)))
        else:
            r = int(_lib.lc_decode_batch_t(self.bp, self.rp, self.ns, self.count, self.sizes, DTYPES[self.dtype], _stream(stream)))
        sizes = list(self.sizes)
        if r < 0 and all(s >= 0 for s in sizes):
            raise LcError(-r)
        return sizes


def lc_decode_batch(blobs, w_refs, stream=None):
    """Restores every tensor from its blob in one call. Returns the list of bytes consumed (negative: -(status))."""
    return DecodeBatch(blobs, w_refs).run(stream)


lc_decode_batch_t = lc_decode_batch      # (DecodeBatch picks the entry point by the tensors' dtype)


CACHE_BYTES = 256


def new_cache(device="cuda"):
    """An empty code table cache for lc_encode_cached."""
    return torch.zeros(CACHE_BYTES, dtype=torch.uint8, device=device)


def lc_encode_cached(w, w_ref, nbits, out, cache, stream=None, n=None):
    """lc_encode with a code table cache (a tensor from new_cache). Returns (blob size, used_cache)."""
    n = w.numel() if n is None else n
    assert out.is_cuda and out.dtype == torch.uint8 and out.is_contiguous()
    assert out.numel() >= lc_encode_bound(n, nbits) > 0 or not (1 <= nbits <= 4), "out is smaller than lc_encode_bound"
    assert cache.is_cuda and cache.dtype == torch.uint8 and cache.is_contiguous() and cache.numel() >= CACHE_BYTES
    used = _int(0)
    r = int(_lib.lc_encode_cached(_dev_f32(w), _dev_f32(w_ref), n, nbits, ctypes.c_void_p(out.data_ptr()),
                                  ctypes.c_void_p(cache.data_ptr()), ctypes.byref(used), _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r, bool(used.value)


def lc_encode_cached_t(w, w_ref, nbits, out, cache, stream=None, n=None):
    """lc_encode_cached for float32, bfloat16 or float16 parameters (w and w_ref of the same dtype)."""
    n = w.numel() if n is None else n
    assert w.dtype == w_ref.dtype
    assert out.is_cuda and out.dtype == torch.uint8 and out.is_contiguous()
    assert out.numel() >= lc_encode_bound(n, nbits) > 0 or not (1 <= nbits <= 4), "out is smaller than lc_encode_bound"
    assert cache.is_cuda and cache.dtype == torch.uint8 and cache.is_contiguous() and cache.numel() >= CACHE_BYTES
    used = _int(0)
    r = int(_lib.lc_encode_cached_t(_dev_any(w), _dev_any(w_ref), n, nbits, ctypes.c_void_p(out.data_ptr()), DTYPES[w.dtype],
                                    ctypes.c_void_p(cache.data_ptr()), ctypes.byref(used), _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r, bool(used.value)


def lc_encode_async_t(w, w_ref, nbits, out, cache=None, stream=None, n=None):
    """lc_encode_async for float32, bfloat16 or float16 parameters."""
    n = w.numel() if n is None else n
    assert w.dtype == w_ref.dtype
    assert out.is_cuda and out.dtype == torch.uint8 and out.is_contiguous()
    assert out.numel() >= lc_encode_bound(n, nbits) > 0 or not (1 <= nbits <= 4), "out is smaller than lc_encode_bound"
    c = None
    if cache is not None:
        assert cache.is_cuda and cache.dtype == torch.uint8 and cache.is_contiguous() and cache.numel() >= CACHE_BYTES
        c = ctypes.c_void_p(cache.data_ptr())
    r = int(_lib.lc_encode_async_t(_dev_any(w), _dev_any(w_ref), n, nbits, ctypes.c_void_p(out.data_ptr()), DTYPES[w.dtype], c,
                                   _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r


def lc_encode_async(w, w_ref, nbits, out, cache=None, stream=None, n=None):
    """Enqueues lc_encode (or lc_encode_cached if `cache` is given) and returns a ticket at once."""
    n = w.numel() if n is None else n
    assert out.is_cuda and out.dtype == torch.uint8 and out.is_contiguous()
    assert out.numel() >= lc_encode_bound(n, nbits) > 0 or not (1 <= nbits <= 4), "out is smaller than lc_encode_bound"
    c = None
    if cache is not None:
        assert cache.is_cuda and cache.dtype == torch.uint8 and cache.is_contiguous() and cache.numel() >= CACHE_BYTES
        c = ctypes.c_void_p(cache.data_ptr())
    r = int(_lib.lc_encode_async(_dev_f32(w), _dev_f32(w_ref), n, nbits, ctypes.c_void_p(out.data_ptr()), c, _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r


def lc_encode_release_inputs(ticket, stream=None):
    """Work enqueued on `stream` after this waits until the call has read w and w_ref for the last time."""
    r = int(_lib.lc_encode_release_inputs(ticket, _stream(stream)))
    if r != 0:
        raise LcError(r)


def lc_encode_wait(ticket):
    """Blocks until the call has finished. Returns (blob size, used_cache)."""
    used = _int(0)
    r = int(_lib.lc_encode_wait(ticket, ctypes.byref(used)))
    if r < 0:
        raise LcError(-r)
    return r, bool(used.value)


def lc_verify(blob, n, dtype=torch.float32, stream=None, blob_bytes=None):
    """Checks a blob from end to end (header, tables, offsets, every lane string) without touching any parameters;
    returns the blob's size in bytes; raises LcError on a negative status."""
    assert blob.is_cuda and blob.dtype == torch.uint8 and blob.is_contiguous()
    size = blob.numel() if blob_bytes is None else blob_bytes
    r = int(_lib.lc_verify(ctypes.c_void_p(blob.data_ptr()), size, n, DTYPES[dtype], _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r


def lc_decode(blob, w_ref, stream=None, n=None):
    """Updates w_ref in place; returns the bytes consumed; raises LcError on a negative status."""
    n = w_ref.numel() if n is None else n
    assert blob.is_cuda and blob.dtype == torch.uint8 and blob.is_contiguous()
    r = int(_lib.lc_decode(ctypes.c_void_p(blob.data_ptr()), _dev_f32(w_ref), n, _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r


def lc_decode_many(blobs, w_ref, stream=None, n=None):
    """Applies the blobs (a list of CUDA uint8 tensors) to w_ref in order; returns the bytes consumed."""
    n = w_ref.numel() if n is None else n
    for b in blobs:
        assert b.is_cuda and b.dtype == torch.uint8 and b.is_contiguous()
    ptrs = (_vp * len(blobs))(*[b.data_ptr() for b in blobs])
    r = int(_lib.lc_decode_many(ptrs, len(blobs), _dev_f32(w_ref), n, _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r


def lc_decode_many_t(blobs, w_ref, stream=None, n=None):
    """lc_decode_many for float32, bfloat16 or float16 parameters."""
    n = w_ref.numel() if n is None else n
    for b in blobs:
        assert b.is_cuda and b.dtype == torch.uint8 and b.is_contiguous()
    ptrs = (_vp * len(blobs))(*[b.data_ptr() for b in blobs])
    r = int(_lib.lc_decode_many_t(ptrs, len(blobs), _dev_any(w_ref), n, DTYPES[w_ref.dtype], _stream(stream)))
    if r < 0:
        raise LcError(-r)
    return r


def lc_blob_info(host_header):
    """host_header: bytes-like, at least 64 bytes, in host memory."""
    buf = (ctypes.c_uint8 * 64).from_buffer_copy(bytes(host_header[:64]))
    n, nbits, total, status = _u64(), _int(), _u64(), _int()
    st = int(_lib.lc_blob_info(buf, ctypes.byref(n), ctypes.byref(nbits), ctypes.byref(total), ctypes.byref(status)))
    if st != OK:
        raise LcError(st)
    return dict(n=n.value, nbits=nbits.value, total_bytes=total.value, status=status.value)


def lc_shutdown():
    _lib.lc_shutdown()


def lc_profile(enable):
    st = int(_lib.lc_profile(1 if enable else 0))
    if st != OK:
        raise LcError(st)


def lc_profile_read():
    """{kernel name: (total ms, launches)} since lc_profile(True)."""
    k = int(_lib.lc_profile_read(None, None, 0))
    ms = (ctypes.c_double * k)()
    cnt = (_u64 * k)()
    _lib.lc_profile_read(ms, cnt, k)
    return {_lib.lc_profile_name(i).decode(): (ms[i], int(cnt[i])) for i in range(k)}


def alloc_out(n, nbits, device="cuda"):
    """A device buffer large enough for any blob of (n, nbits)."""
    return torch.empty(lc_encode_bound(n, nbits), dtype=torch.uint8, device=device)


# ---------------------------------------------------------------- serving a restored checkpoint (include/lc_serve.h)
# `stream` (None: the current one) is where a call's work is enqueued, and nothing else is waited for.  On another stream than the current one the
# caller sees to it that inputs, and an `out` or `ws` that is given, are ready there, and keeps them until that stream is done with them (or calls
# their record_stream).  What a call allocates belongs to `stream`: the current stream, or any other, has to wait for it before it uses the result.
SERVED = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def lc_w4_row_bytes(k):
    """Bytes of a row of k 4-bit codes (a multiple of 16)."""
    return int(_lib.lc_w4_row_bytes(k))


class W4:
    """A matrix [n][k] in 4 bits with group scales: codes uint8 [n][at least lc_w4_row_bytes(k)], scales bfloat16
    [n][at least ceil(k / group)], rows of any pitch (codes: a multiple of 16 bytes).  Keeps the two tensors and the
    marshalled description of them for the calls that take it; they must stay in place."""

    def __init__(self, codes, scales, k, group):
        if group not in (32, 64, 128):
            raise LcError(ERR_BADARG)
        assert codes.is_cuda and codes.dtype == torch.uint8 and codes.dim() == 2 and (codes.stride(1) == 1 or codes.shape[1] <= 1)
        assert scales.is_cuda and scales.dtype == torch.bfloat16 and scales.dim() == 2 and (scales.stride(1) == 1 or scales.shape[1] <= 1)
        assert codes.shape[0] == scales.shape[0] and codes.shape[1] >= lc_w4_row_bytes(k) and scales.shape[1] >= -(-k // group)
        one = codes.shape[0] == 1                            # (the pitch of a single row says nothing)
        self._describe(codes, scales, codes.shape[0], k, group, lc_w4_row_bytes(k) if one else codes.stride(0), scales.shape[1] if one else scales.stride(0))

    def _describe(self, codes, scales, n, k, group, codes_pitch, scales_pitch):
        self.codes, self.scales, self.n, self.k, self.group = codes, scales, n, k, group
        self._c = _W4(codes.data_ptr() or None, scales.data_ptr() or None, n, k, codes_pitch, scales_pitch, group)
        self._p = ctypes.addressof(self._c)


def _handle(stream):
    """_stream for the calls below, which are made once a token: a plain number."""
    if stream is None and _raw_current_stream is not None:
        return _raw_current_stream(_current_device())
    return _stream(stream).value


def _matrix(t):
    """Pointer and pitch of a two-dimensional CUDA tensor whose rows are contiguous."""
    assert t.is_cuda and t.dtype in SERVED and t.dim() == 2, "need a CUDA float32 / bfloat16 / float16 matrix"
    n, k = t.shape
    assert t.stride(1) == 1 or k <= 1, "need contiguous rows"
    return t.data_ptr(), (t.stride(0) if n > 1 else k)


# The calls below have no backward pass: where a gradient is asked for through one it is refused, instead of a result that none flows through.
_NO_GRADIENT = "no gradient flows through this call: detach its inputs, or call it under torch.no_grad()"


def _torch_stream(stream):
    if isinstance(stream, torch.cuda.Stream):
        return stream
    handle = _handle(stream)
    return torch.cuda.ExternalStream(handle) if handle else torch.cuda.default_stream()


def _made_on(stream, make):
    """What make() allocates for a call on `stream`, which need not be the current one: from that stream's memory, since a block of the current one's
    may still be in use by what is enqueued there, which `stream` does not wait for.  Freed, it waits for the current stream's work too, where
    the caller is most likely to use it."""
    s, now = _torch_stream(stream), torch.cuda.current_stream()
    if s == now:
        return make()
    torch.cuda.set_stream(s)                                 # (the context manager for it takes 6 us more)
    try:
        made = make()
    finally:
        torch.cuda.set_stream(now)
    for t in made:
        t.record_stream(now)
    return made


def lc_w4_quantize(w, group, out=None, stream=None):
    """w [n][k] (float32, bfloat16 or float16, contiguous rows) in 4 bits; returns a W4 (`out`, if one is given)."""
    p, ld = _matrix(w)
    n, k = w.shape
    if out is None:
        if group not in (32, 64, 128):
            raise LcError(ERR_BADARG)
        row, groups, device = (k + 31) // 32 * 16, -(-k // group), w.device
        make = lambda: (torch.empty(n, row, dtype=torch.uint8, device=device), torch.empty(n, groups, dtype=torch.bfloat16, device=device))
        codes, scales = make() if stream is None else _made_on(stream, make)
        out = W4.__new__(W4)
        out._describe(codes, scales, n, k, group, row, groups)
    else:
        assert out.n == n and out.k == k and out.group == group
    st = _lib.lc_w4_quantize(p, ld, SERVED[w.dtype], out._p, _handle(stream))
    if st != OK:
        raise LcError(st)
    return out


def lc_w4_dequantize(w4, dtype=None, out=None, stream=None):
    """The values that w4 stands for, as a matrix of `dtype` (or in `out`)."""
    if out is None:
        dtype = torch.float32 if dtype is None else dtype
        make = lambda: (torch.empty(w4.n, w4.k, dtype=dtype, device=w4.codes.device),)
        out, = make() if stream is None else _made_on(stream, make)
        p, ld = out.data_ptr(), w4.k
    else:
        p, ld = _matrix(out)
        assert out.shape == (w4.n, w4.k) and (dtype is None or out.dtype == dtype)
        dtype = out.dtype
    st = _lib.lc_w4_dequantize(w4._p, p, ld, SERVED.get(dtype, -1), _handle(stream))
    if st != OK:
        raise LcError(st)
    return out


def lc_w4_matmul(x, w4, bias=None, out=None, stream=None):
    """x [m][k] times w4 [n][k] transposed, plus bias [n]: a matrix [m][n] of x's dtype (or in `out`).  No gradient flows through it."""
    p, ld = _matrix(x)
    m, k = x.shape
    dtype, n = x.dtype, w4.n
    assert k == w4.k
    assert not x.requires_grad or not torch.is_grad_enabled(), _NO_GRADIENT
    if bias is not None:
        assert not bias.requires_grad or not torch.is_grad_enabled(), _NO_GRADIENT
        assert bias.is_cuda and bias.dtype == dtype and bias.shape == (n,) and (bias.stride(0) == 1 or n <= 1)
        bias = bias.data_ptr()
    if out is None:
        out = x.new_empty(m, n) if stream is None else _made_on(stream, lambda: (x.new_empty(m, n),))[0]
        q, ldq = out.data_ptr(), n
    else:
        q, ldq = _matrix(out)
        assert out.shape == (m, n) and out.dtype == dtype
    st = _lib.lc_w4_matmul(p, ld, m, w4._p, bias, q, ldq, SERVED[dtype], _handle(stream))
    if st != OK:
        raise LcError(st)
    return out


class KvCache:
    """A paged cache of keys and values: k and v uint8 [pages][heads][page_tokens][dim * bits / 8], k_scale and v_scale float32
    [pages][heads][page_tokens], all contiguous.  Keeps the tensors and their marshalled description; they must stay in place."""

    def __init__(self, k, v, k_scale, v_scale, bits):
        if bits not in (8, 4):
            raise LcError(ERR_BADARG)
        for t in (k, v):
            assert t.is_cuda and t.dtype == torch.uint8 and t.dim() == 4 and t.is_contiguous() and t.shape == k.shape
        for t in (k_scale, v_scale):
            assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.shape == k.shape[:3]
        self.k, self.v, self.k_scale, self.v_scale, self.bits = k, v, k_scale, v_scale, bits
        self.pages, self.heads, self.page_tokens, row = k.shape
        self.dim = row * 8 // bits
        self._c = _KvCache(k.data_ptr() or None, v.data_ptr() or None, k_scale.data_ptr() or None, v_scale.data_ptr() or None, self.pages,
                           self.page_tokens, self.heads, self.dim, bits)
        self._p = ctypes.addressof(self._c)


def new_kv_cache(pages, heads, page_tokens, dim, bits, device="cuda"):
    """An empty cache (every key and value zero)."""
    k, v = (torch.full((pages, heads, page_tokens, dim * bits // 8), 0 if bits == 8 else 0x88, dtype=torch.uint8, device=device) for _ in range(2))
    ks, vs = (torch.zeros(pages, heads, page_tokens, dtype=torch.float32, device=device) for _ in range(2))
    return KvCache(k, v, ks, vs, bits)


def _vectors(cache, k, v):
    """Pitches of two tensors [tokens][heads][dim] that are laid out alike, each head's elements contiguous."""
    assert k.is_cuda and v.is_cuda and k.dtype in SERVED and v.dtype == k.dtype and k.dim() == 3 and v.shape == k.shape
    tokens, heads, dim = k.shape
    assert heads == cache.heads and dim == cache.dim
    (st, sh, s1), (vt, vh, v1) = k.stride(), v.stride()      # (the pitch of an axis of one element says nothing)
    assert tokens == 0 or s1 == v1 == 1 and (st == vt or tokens == 1) and (sh == vh or heads == 1), "keys and values need contiguous heads and the same pitches"
    return (st if tokens > 1 else heads * dim), (sh if heads > 1 else dim)


def _slots(slots, tokens):
    assert slots.is_cuda and slots.dtype == torch.int64 and slots.shape == (tokens,) and slots.is_contiguous()
    return slots.data_ptr()


def lc_kv_write(cache, k, v, slots, stream=None):
    """Quantises k and v [tokens][heads][dim] into the cache at `slots` (int64 [tokens]; a negative one is passed over)."""
    ldt, ldh = _vectors(cache, k, v)
    assert not (k.requires_grad or v.requires_grad) or not torch.is_grad_enabled(), _NO_GRADIENT
    tokens = k.shape[0]
    st = _lib.lc_kv_write(cache._p, k.data_ptr(), v.data_ptr(), ldt, ldh, _slots(slots, tokens), tokens, SERVED[k.dtype], _handle(stream))
    if st != OK:
        raise LcError(st)


def lc_kv_read(cache, slots, dtype=None, out=None, stream=None):
    """The keys and values [tokens][heads][dim] that the cache holds at `slots` (zeros for a slot outside), of `dtype` or in out = (k, v)."""
    tokens = slots.shape[0]
    if out is None:
        heads, dim, dtype = cache.heads, cache.dim, torch.float32 if dtype is None else dtype
        make = lambda: (torch.empty(tokens, heads, dim, dtype=dtype, device=slots.device), torch.empty(tokens, heads, dim, dtype=dtype, device=slots.device))
        k, v = make() if stream is None else _made_on(stream, make)
        ldt, ldh = heads * dim, dim
    else:
        k, v = out
        assert k.shape[0] == tokens and (dtype is None or k.dtype == dtype)
        ldt, ldh = _vectors(cache, k, v)
        dtype = k.dtype
    st = _lib.lc_kv_read(cache._p, _slots(slots, tokens), tokens, k.data_ptr(), v.data_ptr(), ldt, ldh, SERVED.get(dtype, -1), _handle(stream))
    if st != OK:
        raise LcError(st)
    return k, v


def lc_kv_workspace_bytes(batch, nq, heads, kv_heads, dim):
    return int(_lib.lc_kv_workspace_bytes(batch, nq, heads, kv_heads, dim))


def new_kv_workspace(cache, batch, nq, heads, stream=None):
    """Scratch for lc_kv_attend with these sizes, to be used on `stream` (None: the current one); calls that may run at the same time need one each."""
    make = lambda: (torch.empty(lc_kv_workspace_bytes(batch, nq, heads, cache.heads, cache.dim), dtype=torch.uint8, device=cache.k.device),)
    return (make() if stream is None else _made_on(stream, make))[0]


def lc_kv_attend(cache, q, table, lens, scale=None, mask=None, out=None, ws=None, stream=None):
    """Attention of q [batch][nq][heads][dim] over the cache: table int32 [batch][pages a sequence], lens int32 [batch] (the nq
    newest tokens are the drafted ones), mask int64 [batch][nq] of the bits that each drafted token sees (None: itself and
    those before it).  scale: 1 / sqrt(dim) if None.  ws: a tensor from new_kv_workspace (None: allocated for this call).  No gradient flows through it."""
    batch, nq, heads, dim = q.shape
    assert q.is_cuda and q.dtype in SERVED and q.is_contiguous() and dim == cache.dim
    assert not q.requires_grad or not torch.is_grad_enabled(), _NO_GRADIENT
    assert table.is_cuda and table.dtype == torch.int32 and table.dim() == 2 and table.shape[0] == batch and (table.stride(1) == 1 or table.shape[1] <= 1)
    assert lens.is_cuda and lens.dtype == torch.int32 and lens.shape == (batch,) and lens.is_contiguous()
    if mask is not None:
        assert mask.is_cuda and mask.dtype == torch.int64 and mask.shape == (batch, nq) and mask.is_contiguous()
        mask = mask.data_ptr()
    if out is None:
        out = torch.empty_like(q) if stream is None else _made_on(stream, lambda: (torch.empty_like(q),))[0]
    else:
        assert out.is_cuda and out.dtype == q.dtype and out.shape == q.shape and out.is_contiguous()
    if ws is None:
        ws = new_kv_workspace(cache, batch, nq, heads, stream)
    assert ws.is_cuda and ws.dtype == torch.uint8 and ws.is_contiguous()
    st = _lib.lc_kv_attend(cache._p, q.data_ptr(), batch, nq, heads, table.data_ptr(), table.stride(0) if batch > 1 else table.shape[1], table.shape[1],
                           lens.data_ptr(), mask, dim ** -0.5 if scale is None else scale, out.data_ptr(), SERVED[q.dtype], ws.data_ptr(), ws.numel(),
                           _handle(stream))
    if st != OK:
        raise LcError(st)
    return out


def lc_i8_workspace_bytes(m, k):
    return int(_lib.lc_i8_workspace_bytes(m, k))


class I8:
    """A matrix [n][k] in 8 bits with a scale a row: codes int8 [n][at least k rounded up to 16], rows of any pitch that is a multiple of 16 bytes, scales float32 [n].
    Keeps the two tensors and their marshalled description; they must stay in place.  Where it is the left side of a product, codes behind k have to be zeros."""

    def __init__(self, codes, scales, k):
        assert codes.is_cuda and codes.dtype == torch.int8 and codes.dim() == 2 and (codes.stride(1) == 1 or codes.shape[1] <= 1)
        assert scales.is_cuda and scales.dtype == torch.float32 and scales.shape == (codes.shape[0],) and (scales.stride(0) == 1 or codes.shape[0] <= 1)
        assert codes.shape[1] >= (k + 15) // 16 * 16
        self._describe(codes, scales, codes.shape[0], k, (k + 15) // 16 * 16 if codes.shape[0] <= 1 else codes.stride(0))

    def _describe(self, codes, scales, n, k, pitch):
        self.codes, self.scales, self.n, self.k = codes, scales, n, k
        self._c = _I8(codes.data_ptr() or None, scales.data_ptr() or None, n, k, pitch)
        self._p = ctypes.addressof(self._c)


def lc_i8_quantize(w, out=None, stream=None):
    """w [n][k] (float32, bfloat16 or float16, contiguous rows) in 8 bits with a scale a row; returns an I8 (`out`, if one is given)."""
    p, ld = _matrix(w)
    n, k = w.shape
    assert not w.requires_grad or not torch.is_grad_enabled(), _NO_GRADIENT
    if out is None:
        row, device = (k + 15) // 16 * 16, w.device
        make = lambda: (torch.empty(n, row, dtype=torch.int8, device=device), torch.empty(n, dtype=torch.float32, device=device))
        codes, scales = make() if stream is None else _made_on(stream, make)
        out = I8.__new__(I8)
        out._describe(codes, scales, n, k, row)
    else:
        assert out.n == n and out.k == k
    st = _lib.lc_i8_quantize(p, ld, SERVED[w.dtype], out._p, _handle(stream))
    if st != OK:
        raise LcError(st)
    return out


def lc_i8_dequantize(w8, dtype=None, out=None, stream=None):
    """The values that w8 stands for, as a matrix of `dtype` (or in `out`)."""
    if out is None:
        dtype = torch.float32 if dtype is None else dtype
        make = lambda: (torch.empty(w8.n, w8.k, dtype=dtype, device=w8.codes.device),)
        out, = make() if stream is None else _made_on(stream, make)
        p, ld = out.data_ptr(), w8.k
    else:
        p, ld = _matrix(out)
        assert out.shape == (w8.n, w8.k) and (dtype is None or out.dtype == dtype)
        dtype = out.dtype
    st = _lib.lc_i8_dequantize(w8._p, p, ld, SERVED.get(dtype, -1), _handle(stream))
    if st != OK:
        raise LcError(st)
    return out


def _bias(bias, n, dtype):
    assert not bias.requires_grad or not torch.is_grad_enabled(), _NO_GRADIENT
    assert bias.is_cuda and bias.dtype == dtype and bias.shape == (n,) and (bias.stride(0) == 1 or n <= 1)
    return bias.data_ptr()


def lc_i8_matmul(x8, w8, bias=None, dtype=None, out=None, stream=None):
    """x8 [m][k] times w8 [n][k] transposed, plus bias [n]: a matrix [m][n] of `dtype` (float32 if None), or in `out`."""
    assert x8.k == w8.k
    m, n = x8.n, w8.n
    if out is None:
        dtype = torch.float32 if dtype is None else dtype
        make = lambda: (torch.empty(m, n, dtype=dtype, device=w8.codes.device),)
        out, = make() if stream is None else _made_on(stream, make)
        q, ldq = out.data_ptr(), n
    else:
        q, ldq = _matrix(out)
        assert out.shape == (m, n) and (dtype is None or out.dtype == dtype)
        dtype = out.dtype
    st = _lib.lc_i8_matmul(x8._p, w8._p, None if bias is None else _bias(bias, n, dtype), q, ldq, SERVED.get(dtype, -1), _handle(stream))
    if st != OK:
        raise LcError(st)
    return out


def new_i8_workspace(m, k, device="cuda", stream=None):
    """Scratch for lc_i8_linear of up to m rows of up to k elements, to be used on `stream` (None: the current one); calls that may run at the same time
    need one each."""
    make = lambda: (torch.empty(lc_i8_workspace_bytes(m, k), dtype=torch.uint8, device=device),)
    return (make() if stream is None else _made_on(stream, make))[0]


def lc_i8_linear(x, w8, bias=None, out=None, ws=None, stream=None):
    """x [m][k] (float32, bfloat16 or float16) times w8 [n][k] transposed, plus bias [n]: a matrix [m][n] of x's dtype (or in `out`), x's rows in 8 bits as by
    lc_i8_quantize.  ws: a tensor from new_i8_workspace (None: allocated for this call).  No gradient flows through it."""
    p, ld = _matrix(x)
    m, k = x.shape
    dtype, n = x.dtype, w8.n
    assert k == w8.k
    assert not x.requires_grad or not torch.is_grad_enabled(), _NO_GRADIENT
    if out is None:
        out = x.new_empty(m, n) if stream is None else _made_on(stream, lambda: (x.new_empty(m, n),))[0]
        q, ldq = out.data_ptr(), n
    else:
        q, ldq = _matrix(out)
        assert out.shape == (m, n) and out.dtype == dtype
    if ws is None:
        ws = new_i8_workspace(m, k, x.device, stream)
    assert ws.is_cuda and ws.dtype == torch.uint8 and ws.is_contiguous()
    st = _lib.lc_i8_linear(p, ld, m, w8._p, None if bias is None else _bias(bias, n, dtype), q, ldq, SERVED[dtype], ws.data_ptr(), ws.numel(), _handle(stream))
    if st != OK:
        raise LcError(st)
    return out


def lc_kv_prompt_workspace_bytes(tokens, batch, heads, kv_heads, dim):
    return int(_lib.lc_kv_prompt_workspace_bytes(tokens, batch, heads, kv_heads, dim))


def lc_kv_prompt_workspace_most(tokens, batch, heads, kv_heads, dim):
    return int(_lib.lc_kv_prompt_workspace_most(tokens, batch, heads, kv_heads, dim))


def new_prompt_workspace(cache, tokens, batch, heads, stream=None):
    """Scratch for lc_kv_attend_prompt of up to `tokens` new tokens of up to `batch` sequences, to be used on `stream` (None: the current one); calls that may run at the
    same time need one each."""
    make = lambda: (torch.empty(lc_kv_prompt_workspace_most(tokens, batch, heads, cache.heads, cache.dim), dtype=torch.uint8, device=cache.k.device),)
    return (make() if stream is None else _made_on(stream, make))[0]


def _tokens_of(t):
    """Pitch of a tensor [tokens][heads][dim] whose tokens are contiguous."""
    assert t.is_cuda and t.dtype in SERVED and t.dim() == 3, "need a CUDA float32 / bfloat16 / float16 tensor [tokens][heads][dim]"
    tokens, heads, dim = t.shape
    (st, sh, s1) = t.stride()
    assert tokens == 0 or (s1 == 1 and (sh == dim or heads == 1)), "need contiguous tokens"
    return st if tokens > 1 else heads * dim


def lc_kv_attend_prompt(cache, q, starts, table, lens, scale=None, out=None, ws=None, stream=None):
    """Attention of the new tokens of several sequences over the cache: q [tokens][heads][dim], of sequence b those from starts[b] to before starts[b + 1] (int32
    [batch + 1], not decreasing), which are the newest of its lens[b] cached ones and see what is cached up to themselves; table and lens as for lc_kv_attend.
    scale: 1 / sqrt(dim) if None.  ws: a tensor from new_prompt_workspace (None: allocated for this call).  Rows of `out` (None: a new tensor) that no sequence
    has are left as they are.  No gradient flows through it."""
    ldq = _tokens_of(q)
    tokens, heads, dim = q.shape
    assert dim == cache.dim
    assert not q.requires_grad or not torch.is_grad_enabled(), _NO_GRADIENT
    batch = lens.shape[0]
    assert starts.is_cuda and starts.dtype == torch.int32 and starts.shape == (batch + 1,) and starts.is_contiguous()
    assert table.is_cuda and table.dtype == torch.int32 and table.dim() == 2 and table.shape[0] == batch and (table.stride(1) == 1 or table.shape[1] <= 1)
    assert lens.is_cuda and lens.dtype == torch.int32 and lens.dim() == 1 and lens.is_contiguous()
    if out is None:
        make = lambda: (torch.empty(tokens, heads, dim, dtype=q.dtype, device=q.device),)
        out, = make() if stream is None else _made_on(stream, make)
        ldo = heads * dim
    else:
        assert out.dtype == q.dtype and out.shape == q.shape
        ldo = _tokens_of(out)
    if ws is None:
        make = lambda: (torch.empty(lc_kv_prompt_workspace_bytes(tokens, batch, heads, cache.heads, dim), dtype=torch.uint8, device=q.device),)
        ws, = make() if stream is None else _made_on(stream, make)
    assert ws.is_cuda and ws.dtype == torch.uint8 and ws.is_contiguous()
    st = _lib.lc_kv_attend_prompt(cache._p, q.data_ptr(), ldq, tokens, heads, starts.data_ptr(), batch, table.data_ptr(),
                                  table.stride(0) if batch > 1 else table.shape[1], table.shape[1], lens.data_ptr(), dim ** -0.5 if scale is None else scale,
                                  out.data_ptr(), ldo, SERVED[q.dtype], ws.data_ptr(), ws.numel(), _handle(stream))
    if st != OK:
        raise LcError(st)
    return out


class KvPages:
    """The pages of sequences that share a cache: table int32 [batch][pages a sequence] and lens int32 [batch], which attention takes, free_pages int32 [room], a stack
    of the pages that nobody has, and free_count int32 [1], how many there are.  Keeps the tensors and their marshalled description; they must stay in place."""

    def __init__(self, table, lens, free_pages, free_count, page_tokens):
        batch = lens.shape[0]
        assert table.is_cuda and table.dtype == torch.int32 and table.dim() == 2 and table.shape[0] == batch and (table.stride(1) == 1 or table.shape[1] <= 1)
        for t in (lens, free_pages, free_count):
            assert t.is_cuda and t.dtype == torch.int32 and t.dim() == 1 and t.is_contiguous()
        assert free_count.shape == (1,)
        self.table, self.lens, self.free_pages, self.free_count, self.page_tokens, self.batch = table, lens, free_pages, free_count, page_tokens, batch
        self._c = _KvPages(table.data_ptr() or None, lens.data_ptr() or None, free_pages.data_ptr() or None, free_count.data_ptr(), batch,
                           table.stride(0) if batch > 1 else table.shape[1], table.shape[1], free_pages.shape[0], page_tokens)
        self._p = ctypes.addressof(self._c)


def new_kv_pages(cache, batch, context):
    """The pages of `batch` empty sequences of up to `context` tokens each that share all of the cache; page 0 is given out first."""
    device = cache.k.device
    table = torch.zeros(batch, -(-context // cache.page_tokens), dtype=torch.int32, device=device)
    return KvPages(table, torch.zeros(batch, dtype=torch.int32, device=device), torch.arange(cache.pages - 1, -1, -1, dtype=torch.int32, device=device),
                   torch.full((1,), cache.pages, dtype=torch.int32, device=device), cache.page_tokens)


def _counts(t, n):
    assert t.is_cuda and t.dtype == torch.int32 and t.shape == (n,) and t.is_contiguous()
    return t.data_ptr()


def lc_kv_extend(pages, add, room, new_lens=None, new_count=None, out=None, stream=None):
    """Room for add[b] (int32 [batch]) more tokens of each sequence, of all sequences together at most `room`; the leading sequences for which pages, their rows of the
    table and `room` suffice get theirs.  Returns starts int32 [batch + 1], and of the new tokens slots int64 [room], places and owners int32 [room] (-1 behind the
    last), in out = (starts, slots, places, owners) if given.  The lengths and the number of free pages go to new_lens and new_count (None: into `pages`)."""
    batch, device = pages.batch, pages.lens.device
    if out is None:
        make = lambda: (torch.empty(room, dtype=torch.int64, device=device), torch.empty(batch + 1, dtype=torch.int32, device=device),
                        torch.empty(2, room, dtype=torch.int32, device=device))
        slots, starts, both = make() if stream is None else _made_on(stream, make)
        places, owners = both.unbind(0)
    else:
        starts, slots, places, owners = out
        assert slots.is_cuda and slots.dtype == torch.int64 and slots.shape == (room,) and slots.is_contiguous()
        _counts(starts, batch + 1), _counts(places, room), _counts(owners, room)
    st = _lib.lc_kv_extend(pages._p, _counts(add, batch), room, pages.lens.data_ptr() if new_lens is None else _counts(new_lens, batch),
                           pages.free_count.data_ptr() if new_count is None else _counts(new_count, 1), starts.data_ptr(), slots.data_ptr(), places.data_ptr() or None,
                           owners.data_ptr() or None, _handle(stream))
    if st != OK:
        raise LcError(st)
    return starts, slots, places, owners


def lc_kv_trim(pages, keep, new_lens=None, new_count=None, stream=None):
    """Of every sequence its first keep[b] tokens stay (int32 [batch]), and the pages behind them go back on the stack.  The lengths and the number of free pages go to
    new_lens and new_count (None: into `pages`)."""
    st = _lib.lc_kv_trim(pages._p, _counts(keep, pages.batch), pages.lens.data_ptr() if new_lens is None else _counts(new_lens, pages.batch),
                         pages.free_count.data_ptr() if new_count is None else _counts(new_count, 1), _handle(stream))
    if st != OK:
        raise LcError(st)


def lc_draft_workspace_bytes(batch):
    return int(_lib.lc_draft_workspace_bytes(batch))


def new_draft_workspace(batch, device="cuda", stream=None):
    """Scratch for lc_draft_verify of up to `batch` sequences, to be used on `stream` (None: the current one); calls that may run at the same time need one each."""
    make = lambda: (torch.empty(lc_draft_workspace_bytes(batch), dtype=torch.uint8, device=device),)
    return (make() if stream is None else _made_on(stream, make))[0]


def _rows(t, batch, rows, vocab):
    """Pitches of probabilities [batch][rows][vocab] whose rows are contiguous."""
    assert t.is_cuda and t.dtype in SERVED and t.shape == (batch, rows, vocab) and (t.stride(2) == 1 or vocab == 1 or t.numel() == 0)
    assert not t.requires_grad or not torch.is_grad_enabled(), _NO_GRADIENT
    return t.data_ptr(), (t.stride(0) if batch > 1 else rows * vocab), (t.stride(1) if rows > 1 else vocab)


def lc_draft_verify(target, tokens, uniform, draft=None, parent=None, count=None, out=None, ws=None, stream=None):
    """Judges drafted tokens against the model's probabilities target [batch][nodes][vocab], those behind each node; tokens int32 [batch][nodes], of which node 0 is known.
    draft [batch][nodes - 1][vocab]: what nodes 1, 2 ... were drawn from, one behind the other; without it they are guesses, below parent int32 [batch][nodes] (None:
    below the one before).  count int32 [batch]: nodes that exist (None: all).  uniform float32 [batch][nodes] in [0, 1): for each node's judgement, and node 0's
    for the token drawn behind the path.  Returns {"path": int32 [batch][nodes], node numbers and -1 behind them, "count": int32 [batch], how many, "next": int32
    [batch], the token drawn}, in out = (path, count, next) if given.  ws: a tensor from new_draft_workspace (None: allocated for this call)."""
    batch, nodes, vocab = target.shape
    p, ldb, ldr = _rows(target, batch, nodes, vocab)
    q, qldb, qldr = (None, 0, 0) if draft is None else _rows(draft, batch, nodes - 1, vocab)
    assert draft is None or draft.dtype == target.dtype
    for t, dtype in ((tokens, torch.int32), (uniform, torch.float32)) if parent is None else ((tokens, torch.int32), (uniform, torch.float32), (parent, torch.int32)):
        assert t.is_cuda and t.dtype == dtype and t.shape == (batch, nodes) and t.is_contiguous()
    if out is None:
        make = lambda: (torch.empty(batch, nodes, dtype=torch.int32, device=target.device), torch.empty(2, batch, dtype=torch.int32, device=target.device))
        path, few = make() if stream is None else _made_on(stream, make)
        length, following = few.unbind(0)
    else:
        path, length, following = out
        assert path.is_cuda and path.dtype == torch.int32 and path.shape == (batch, nodes) and path.is_contiguous()
    if ws is None:
        ws = new_draft_workspace(batch, target.device, stream)
    assert ws.is_cuda and ws.dtype == torch.uint8 and ws.is_contiguous()
    st = _lib.lc_draft_verify(p, ldb, ldr, batch, nodes, vocab, tokens.data_ptr(), q or None, qldb, qldr, None if parent is None else parent.data_ptr(),
                              None if count is None else _counts(count, batch), uniform.data_ptr(), SERVED[target.dtype], path.data_ptr(), _counts(length, batch),
                              _counts(following, batch), ws.data_ptr(), ws.numel(), _handle(stream))
    if st != OK:
        raise LcError(st)
    return {"path": path, "count": length, "next": following}

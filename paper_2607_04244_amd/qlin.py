"""Python binding of ``libqlin.so`` (argument marshalling only).

The functions mirror the C ABI in ``include/qlin.h`` one to one; ``QLinear``
wraps a handle for torch callers.  torch supplies device memory and the
current stream; every step of the computation runs in the HIP kernels.  The
module raises if the library has not been built - there is no fallback.
"""

import ctypes
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# QLIN_LIB selects another build of the same library (the sanitizer build of
# the CPU tests); by default the in-tree libqlin.so
LIB_PATH = os.environ.get("QLIN_LIB") or os.path.join(_HERE, "libqlin.so")

QLIN_OK = 0
QLIN_ERR_INVALID = -1
QLIN_ERR_UNSUPPORTED = -2
QLIN_ERR_ALIGN = -3
QLIN_ERR_OOM = -4
QLIN_ERR_HIP = -5

PATH_AUTO, PATH_GEMV, PATH_SKINNY, PATH_TILED, PATH_REGS = 0, 1, 2, 3, 4

# every symbol include/*.h declare
EXPORTS = ("qlin_create", "qlin_create_symmetric", "qlin_forward", "qlin_forward_path",
           "qlin_plan", "qlin_destroy", "qlin_last_error", "qlin_unpack_codes",
           "qlin_dequantize", "qlin_shape", "qlin_last_status", "qlin_stream_read", "qlin_quantize",
           "qlin_swa_plan", "qlin_swa_attention", "qlin_forward_group", "qlin_group_plan",
           "qlin_workspace_bytes", "qlin_forward_group_noalloc", "qlin_norm_rope_append", "qlin_causal_plan",
           "qlin_causal_attention", "qlin_verify_plan", "qlin_verify_draft")

_lib = None


class Batch(ctypes.Structure):
    """struct qlin_batch (include/qlin_target.h); pointers are device addresses."""
    _fields_ = [("n_seq", ctypes.c_int64), ("rows", ctypes.c_int64), ("max_new", ctypes.c_int64),
                ("max_len", ctypes.c_int64), ("new_start", ctypes.c_void_p), ("length", ctypes.c_void_p),
                ("cache_start", ctypes.c_void_p)]


class _Room(ctypes.Structure):
    _fields_ = [("capacity", ctypes.c_int64)]


class KVCache(_Room):
    """struct qlin_kv_cache (include/qlin_target.h); strides in elements.  Its first member,
    capacity, is given by name, and is 0 (no bound) without."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("heads", ctypes.c_int64), ("slots", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("seq_slots", ctypes.c_int64)]

    def __init__(self, *fields, capacity=0):
        super().__init__(capacity, *fields)


_cache_members = struct.Struct("=8q").pack


class QlinError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"qlin error {code}: {msg}")
        self.code = code


def lib():
    """Load ``libqlin.so`` (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"HIP library {LIB_PATH} is missing: run __graft_entry__.build() first")
    L = ctypes.CDLL(LIB_PATH)
    P, I64, I32, VP = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p
    L.qlin_create.restype = P
    L.qlin_create.argtypes = [I64, I64, I64, VP, VP, VP]
    L.qlin_create_symmetric.restype = P
    L.qlin_create_symmetric.argtypes = [I64, I64, I64, VP, VP]
    L.qlin_quantize.restype = I32
    L.qlin_quantize.argtypes = [I64, I64, I64, VP, VP, VP, VP, VP]
    L.qlin_forward.restype = I32
    L.qlin_forward.argtypes = [P, I64, VP, VP, VP]
    L.qlin_forward_path.restype = I32
    L.qlin_forward_path.argtypes = [P, I32, I64, I64, VP, VP, VP]
    L.qlin_plan.restype = I32
    L.qlin_plan.argtypes = [P, I32, I64, I64, ctypes.c_char_p, I64]
    L.qlin_destroy.restype = None
    L.qlin_destroy.argtypes = [P]
    L.qlin_last_error.restype = ctypes.c_char_p
    L.qlin_last_error.argtypes = []
    L.qlin_last_status.restype = I32
    L.qlin_last_status.argtypes = []
    L.qlin_unpack_codes.restype = I32
    L.qlin_unpack_codes.argtypes = [P, VP, VP]
    L.qlin_dequantize.restype = I32
    L.qlin_dequantize.argtypes = [P, I32, VP, VP]
    L.qlin_stream_read.restype = I32
    L.qlin_stream_read.argtypes = [VP, I64, I32, VP, VP]
    L.qlin_swa_plan.restype = I32
    L.qlin_swa_plan.argtypes = [I64, I64, I64, I64, I64, I64, I64, ctypes.POINTER(I64), ctypes.POINTER(I64),
                                ctypes.c_char_p, I64]
    L.qlin_swa_attention.restype = I32
    L.qlin_swa_attention.argtypes = [I64, I64, I64, I64, I64, I64, I64, I64, VP, VP, VP, VP, VP, I64, VP]
    L.qlin_forward_group.restype = I32
    L.qlin_forward_group.argtypes = [I64, VP, I32, I64, I64, VP, VP, VP, I64, VP]
    L.qlin_forward_group_noalloc.restype = I32
    L.qlin_forward_group_noalloc.argtypes = [I64, VP, I32, I64, I64, VP, VP, VP]
    L.qlin_group_plan.restype = I32
    L.qlin_group_plan.argtypes = [I64, VP, I32, I64, I64, I64, ctypes.POINTER(I64), ctypes.c_char_p, I64]
    L.qlin_workspace_bytes.restype = I32
    L.qlin_workspace_bytes.argtypes = [P, ctypes.POINTER(I64)]
    BP, CP, F32 = ctypes.POINTER(Batch), ctypes.POINTER(KVCache), ctypes.c_float
    L.qlin_norm_rope_append.restype = I32
    L.qlin_norm_rope_append.argtypes = [BP, CP, I64, I64, VP, I64, VP, I64, VP, I64, VP, VP, F32, VP, I64, I32, VP,
                                        I64, VP]
    L.qlin_causal_plan.restype = I32
    L.qlin_causal_plan.argtypes = [BP, I64, I64, I64, I64, ctypes.POINTER(I64), ctypes.POINTER(I64), ctypes.c_char_p,
                                   I64]
    L.qlin_causal_attention.restype = I32
    L.qlin_causal_attention.argtypes = [BP, CP, I64, I64, F32, I64, VP, I64, VP, I64, VP, I64, VP]
    L.qlin_verify_plan.restype = I32
    L.qlin_verify_plan.argtypes = [I64, I64, I64, ctypes.POINTER(I64)]
    L.qlin_verify_draft.restype = I32
    L.qlin_verify_draft.argtypes = [I64, I64, I64, VP, I64, VP, I64, VP, VP, VP, VP, VP, VP, VP, I64, VP]
    L.qlin_shape.restype = I32
    L.qlin_shape.argtypes = [P, ctypes.POINTER(I64), ctypes.POINTER(I64)]
    _lib = L
    return L


def last_error():
    return lib().qlin_last_error().decode()


def qlin_last_error():
    return last_error()


def qlin_last_status():
    return lib().qlin_last_status()


def _check(rc):
    if rc != QLIN_OK:
        raise QlinError(rc, last_error())
    return rc


def _host_ptr(a, dtype):
    """(keep-alive object, address) of a host array, or of a device tensor
    (any object with data_ptr(), passed through as is)."""
    if a is None:
        return None, None
    if hasattr(a, "data_ptr"):
        return a, a.data_ptr()
    a = np.ascontiguousarray(a, dtype=dtype)
    return a, a.ctypes.data


# ---------------------------------------------------------------- C ABI mirror

def qlin_create(K, N, group, packed_w, scales, zeros):
    """Host numpy arrays in; returns the handle (int) or raises QlinError."""
    p, pp = _host_ptr(packed_w, np.uint32)
    s, sp = _host_ptr(scales, np.uint16)
    z, zp = _host_ptr(zeros, np.uint16)
    h = lib().qlin_create(K, N, group, pp, sp, zp)
    if not h:
        raise QlinError(lib().qlin_last_status(), last_error())
    return h


def qlin_create_symmetric(K, N, group, packed_w, scales):
    p, pp = _host_ptr(packed_w, np.uint32)
    s, sp = _host_ptr(scales, np.uint16)
    h = lib().qlin_create_symmetric(K, N, group, pp, sp)
    if not h:
        raise QlinError(lib().qlin_last_status(), last_error())
    return h


def qlin_quantize(K, N, group, w_ptr, scales_ptr, zeros_ptr, packed_ptr, stream):
    return lib().qlin_quantize(K, N, group, w_ptr, scales_ptr, zeros_ptr, packed_ptr, stream)


def quantize(w, scales, zeros=None, group=128):
    """Device bf16 weights [N, K] -> device packed codes (torch.int32 view of
    uint32 words) [N, K/8] on the frozen grid (scales, zeros device bf16
    [N, K/128]; zeros=None is the symmetric format)."""
    import torch
    N, K = w.shape
    w = w.contiguous()
    packed = torch.empty((N, K // 8), dtype=torch.int32, device=w.device)
    zp = zeros.contiguous().data_ptr() if zeros is not None else None
    _check(qlin_quantize(K, N, group, w.data_ptr(), scales.contiguous().data_ptr(), zp, packed.data_ptr(),
                         _stream()))
    return packed


def qlin_forward(h, M, x_ptr, y_ptr, stream):
    return lib().qlin_forward(h, M, x_ptr, y_ptr, stream)


def qlin_forward_path(h, path, split_k, M, x_ptr, y_ptr, stream):
    return lib().qlin_forward_path(h, path, split_k, M, x_ptr, y_ptr, stream)


def qlin_plan(h, path, split_k, M):
    buf = ctypes.create_string_buffer(256)
    _check(lib().qlin_plan(h, path, split_k, M, buf, len(buf)))
    return buf.value.decode()


def _handles(hs):
    arr = (ctypes.c_void_p * len(hs))(*hs)
    return arr


def qlin_forward_group(hs, path, split_k, M, x_ptr, y_ptrs, ws_ptr, ws_bytes, stream):
    """hs: sequence of handles; y_ptrs: sequence of device addresses."""
    ys = (ctypes.c_void_p * len(y_ptrs))(*y_ptrs)
    return lib().qlin_forward_group(len(hs), _handles(hs), path, split_k, M, x_ptr, ys, ws_ptr, ws_bytes, stream)


def qlin_forward_group_noalloc(hs, path, split_k, M, x_ptr, y_ptrs, stream):
    ys = (ctypes.c_void_p * len(y_ptrs))(*y_ptrs)
    return lib().qlin_forward_group_noalloc(len(hs), _handles(hs), path, split_k, M, x_ptr, ys, stream)


def qlin_group_plan(hs, path, split_k, M, ws_bytes=-1):
    """(workspace bytes the plan uses, plan text) for a workspace of ws_bytes (-1: no limit)."""
    need = ctypes.c_int64()
    buf = ctypes.create_string_buffer(256)
    _check(lib().qlin_group_plan(len(hs), _handles(hs), path, split_k, M, ws_bytes, ctypes.byref(need), buf,
                                 len(buf)))
    return need.value, buf.value.decode()


def qlin_workspace_bytes(h):
    b = ctypes.c_int64()
    _check(lib().qlin_workspace_bytes(h, ctypes.byref(b)))
    return b.value


def qlin_destroy(h):
    lib().qlin_destroy(h)


def qlin_unpack_codes(h, q_ptr, stream):
    return lib().qlin_unpack_codes(h, q_ptr, stream)


def qlin_dequantize(h, routine, w_ptr, stream):
    return lib().qlin_dequantize(h, routine, w_ptr, stream)


def qlin_stream_read(buf_ptr, nbytes, grid, sink_ptr, stream):
    return lib().qlin_stream_read(buf_ptr, nbytes, grid, sink_ptr, stream)


def qlin_shape(h):
    K, N = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().qlin_shape(h, ctypes.byref(K), ctypes.byref(N)))
    return K.value, N.value


def qlin_swa_plan(Hq, Hkv, head_dim, nq, T, window, splits=0):
    """(splits, workspace_bytes, text) of the drafter attention's plan."""
    S, ws = ctypes.c_int64(), ctypes.c_int64()
    buf = ctypes.create_string_buffer(256)
    _check(lib().qlin_swa_plan(Hq, Hkv, head_dim, nq, T, window, splits, ctypes.byref(S), ctypes.byref(ws),
                               buf, len(buf)))
    return S.value, ws.value, buf.value.decode()


def qlin_swa_attention(Hq, Hkv, head_dim, nq, T, kv_stride, window, splits, q_ptr, k_ptr, v_ptr, out_ptr,
                       ws_ptr, ws_bytes, stream):
    return lib().qlin_swa_attention(Hq, Hkv, head_dim, nq, T, kv_stride, window, splits, q_ptr, k_ptr, v_ptr,
                                    out_ptr, ws_ptr, ws_bytes, stream)


def qlin_norm_rope_append(batch, cache, q_heads, head_dim, q_ptr, q_stride, k_ptr, k_stride, v_ptr, v_stride,
                          q_norm_ptr, k_norm_ptr, eps, inv_freq_ptr, rotary_dim, interleaved, q_out_ptr, q_out_stride,
                          stream):
    """batch: Batch, cache: KVCache (or None: NULL)."""
    return lib().qlin_norm_rope_append(batch, cache, q_heads, head_dim, q_ptr, q_stride, k_ptr, k_stride, v_ptr,
                                       v_stride, q_norm_ptr, k_norm_ptr, eps, inv_freq_ptr, rotary_dim, interleaved,
                                       q_out_ptr, q_out_stride, stream)


def qlin_causal_plan(batch, q_heads, kv_heads, head_dim, splits=0):
    """(splits, workspace_bytes, text) of the causal attention's plan."""
    S, ws = ctypes.c_int64(), ctypes.c_int64()
    buf = ctypes.create_string_buffer(256)
    _check(lib().qlin_causal_plan(batch, q_heads, kv_heads, head_dim, splits, ctypes.byref(S), ctypes.byref(ws), buf,
                                  len(buf)))
    return S.value, ws.value, buf.value.decode()


def qlin_causal_attention(batch, cache, q_heads, head_dim, scale, splits, q_ptr, q_stride, out_ptr, out_stride, ws_ptr,
                          ws_bytes, stream):
    return lib().qlin_causal_attention(batch, cache, q_heads, head_dim, scale, splits, q_ptr, q_stride, out_ptr,
                                       out_stride, ws_ptr, ws_bytes, stream)


def qlin_verify_plan(n_seq, n_draft, vocab):
    """Workspace bytes of qlin_verify_draft."""
    ws = ctypes.c_int64()
    _check(lib().qlin_verify_plan(n_seq, n_draft, vocab, ctypes.byref(ws)))
    return ws.value


def qlin_verify_draft(n_seq, n_draft, vocab, target_ptr, target_stride, draft_ptr, draft_stride, drafted_ptr, count_ptr,
                      temperature_ptr, uniform_ptr, accepted_ptr, tokens_ptr, ws_ptr, ws_bytes, stream):
    return lib().qlin_verify_draft(n_seq, n_draft, vocab, target_ptr, target_stride, draft_ptr, draft_stride,
                                   drafted_ptr, count_ptr, temperature_ptr, uniform_ptr, accepted_ptr, tokens_ptr,
                                   ws_ptr, ws_bytes, stream)


# ---------------------------------------------------------------- torch wrappers

_raw_stream = _current_device = None


def _stream():
    """The current stream of the current device, as an integer (for callers
    that hold a CUDA tensor or a handle, so CUDA is initialised).  torch's raw
    getters: building a torch.cuda.Stream object to ask it for its pointer
    takes 2.5 us, a quarter of a small call; the getters take 0.1 us."""
    global _raw_stream, _current_device
    if _raw_stream is None:
        import torch
        _current_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    return _raw_stream(_current_device())


def swa_attention(q, k, v, window, T=None, splits=0, out=None, workspace=None):
    """Drafter block attention with a symmetric window (include/qlin_attn.h).

    q: CUDA bf16 [Hq, nq, 128]; k, v: CUDA bf16 [Hkv, capacity, 128] with the
    first T tokens valid (T defaults to the capacity); window 0 = full
    attention.  ``workspace`` (a CUDA tensor of at least the planned bytes) is
    allocated when needed and not given.  Returns ``out`` [Hq, nq, 128].
    """
    import torch
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != 3 or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous CUDA bf16 tensor of rank 3")
    Hq, nq, D = q.shape
    Hkv, cap, _ = k.shape
    if v.shape != k.shape:
        raise ValueError("k and v must have the same shape")
    if k.device != q.device or v.device != q.device:
        raise ValueError("q, k and v must be on one device")
    T = cap if T is None else T
    if workspace is None:                        # with one given, the call itself checks sizes and plan
        _, ws_bytes, _ = qlin_swa_plan(Hq, Hkv, D, nq, T, window, splits)
        if ws_bytes:
            workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=q.device)
    if out is None:
        out = torch.empty((Hq, nq, D), dtype=torch.bfloat16, device=q.device)
    else:
        _check_out(out, (Hq, nq, D), q.device)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_len = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(qlin_swa_attention(Hq, Hkv, D, nq, T, cap, window, splits, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                              out.data_ptr(), ws_ptr, ws_len, _stream()))
    return out


def _check_out(out, shape, device):
    import torch
    if (not isinstance(out, torch.Tensor) or out.dtype != torch.bfloat16 or out.device != device
            or tuple(out.shape) != tuple(shape) or not out.is_contiguous()):
        raise ValueError(f"out must be a contiguous bf16 tensor of shape {tuple(shape)} on {device}")


_torch = None


def _device():
    """The current device's index (and torch loaded, for callers that hold CUDA tensors)."""
    global _torch, _raw_stream, _current_device
    if _torch is None:
        import torch
        _current_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        _torch = torch                                      # last: what the test above goes by, in any thread
    return _current_device()


def _address(name, t, dtype, dev):
    """The address of a tensor, which has to be of this type on the current device (its
    stream's).  The checks of a call cost about as much as its launch: one pass, no
    torch.device objects."""
    try:
        if t.dtype is dtype and t.get_device() == dev:
            return t.data_ptr()
    except AttributeError:                                  # no tensor
        pass
    raise ValueError(f"{name} must be a {dtype} tensor on the current CUDA device")


def _vector(name, t, dtype, dev, n):
    """The address of a contiguous tensor of n values; None stays None."""
    if t is None:
        return None
    p = _address(name, t, dtype, dev)
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous, of {n} values")
    return p


def _kv_cache(k_cache, v_cache, dev):
    """KVCache of [sequences, heads, capacity, 128] or packed [tokens, heads, 128] tensors."""
    k = _address("k_cache", k_cache, _torch.bfloat16, dev)
    v = _address("v_cache", v_cache, _torch.bfloat16, dev)
    shape, stride = k_cache.shape, k_cache.stride()
    if v_cache.shape != shape or v_cache.stride() != stride:
        raise ValueError("k_cache and v_cache must have the same shape and strides")
    rank = len(shape)
    if rank not in (3, 4) or shape[-1] != 128 or stride[-1] != 1 or 0 in shape:
        raise ValueError("the cache must be [sequences, heads, capacity, 128] or [tokens, heads, 128], rows contiguous")
    if rank == 3:
        return KVCache(k, v, shape[1], shape[0], stride[0], stride[1], 0)
    n, heads, capacity, _ = shape
    seq, head, token, _ = stride
    if n == 1:
        seq = 0
    if token <= 0 or seq % token:
        raise ValueError("the cache's sequences must lie whole tokens apart")
    seq //= token
    # the members packed: a third of the constructor's time
    return KVCache.from_buffer_copy(_cache_members(capacity, k, v, heads, (n - 1) * seq + capacity, token, head, seq))


def _batch(dev, rows, new_start, length, max_new, max_len, cache_start, k_cache):
    i32 = _torch.int32
    lengths = _address("length", length, i32, dev)
    n = length.numel()
    if not length.is_contiguous():
        raise ValueError("length must be contiguous")
    starts = _vector("new_start", new_start, i32, dev, n + 1)
    slots = _vector("cache_start", cache_start, _torch.int64, dev, n)
    if slots is None and n > 1 and (k_cache.dim() == 3 or k_cache.shape[0] < n):
        raise ValueError("several sequences need cache_start or a cache of as many sequences")
    if max_len is None:
        max_len = k_cache.shape[-2] if k_cache.dim() == 4 else k_cache.shape[0]
    return Batch(n, rows, rows if max_new is None or max_new > rows else max_new, max_len, starts, lengths, slots)


def _row_stride(name, t, heads):
    """Elements between the rows of [rows, heads, 128], heads contiguous."""
    row, head, one = t.stride()
    if one != 1 or (heads > 1 and head != 128):
        raise ValueError(f"{name}: the heads of a row must be contiguous")
    return row if t.shape[0] > 1 else heads * 128


def norm_rope_append(q, k, v, k_cache, v_cache, new_start, length, max_new=None, max_len=None, cache_start=None,
                     q_norm=None, k_norm=None, eps=1e-6, inv_freq=None, interleaved=False, out=None):
    """Norms and rotation of the new tokens' queries and keys, keys and values
    appended to the cache (qlin_norm_rope_append in include/qlin_target.h).

    q, k, v: CUDA bf16 [rows, heads * 128], row slices allowed; k_cache, v_cache:
    bf16 [sequences, heads, capacity, 128], or packed [tokens, heads, 128] with
    ``cache_start`` (int64, the slot of each sequence's token 0).  new_start int32
    [n + 1] and length int32 [n] describe the sequences' new tokens and cached
    lengths; max_new bounds the new tokens of a sequence.  q_norm, k_norm: bf16 [128]
    or None; inv_freq: float64 [rotary_dim / 2] or None.  Returns ``out`` [rows,
    q heads, 128]; rows of no sequence are left as they are.
    """
    dev = _device()
    bf16 = _torch.bfloat16
    cache = _kv_cache(k_cache, v_cache, dev)
    at, strides, widths = [], [], []
    for name, t in (("q", q), ("k", k), ("v", v)):
        at.append(_address(name, t, bf16, dev))
        shape = t.shape
        if len(shape) != 2:
            raise ValueError(f"{name} must have rank 2")
        (rows, width), (row, one) = shape, t.stride()
        if width == 0 or width % 128 or one != 1 or (widths and rows != q.shape[0]):
            raise ValueError(f"{name} must be [rows, heads * 128] with contiguous rows")
        strides.append(row if rows > 1 else width)
        widths.append(width)
    Hq = widths[0] // 128
    if widths[1] != cache.heads * 128 or widths[2] != widths[1]:
        raise ValueError(f"k and v must have the cache's {cache.heads} heads")
    batch = _batch(dev, rows, new_start, length, max_new, max_len, cache_start, k_cache)
    rotary, freq = 0, None
    if inv_freq is not None:
        half = inv_freq.numel()
        rotary, freq = 2 * half, _vector("inv_freq", inv_freq, _torch.float64, dev, half)
    if out is None:
        out = _torch.empty((rows, Hq, 128), dtype=bf16, device=q.device)
        out_at, out_stride = out.data_ptr(), widths[0]
    else:
        out_at = _address("out", out, bf16, dev)
        if out.shape != (rows, Hq, 128):
            raise ValueError(f"out must have shape {(rows, Hq, 128)}")
        out_stride = _row_stride("out", out, Hq)
    _check(lib().qlin_norm_rope_append(batch, cache, Hq, 128, at[0], strides[0], at[1], strides[1], at[2], strides[2],
                                       _vector("q_norm", q_norm, bf16, dev, 128),
                                       _vector("k_norm", k_norm, bf16, dev, 128), eps, freq, rotary,
                                       1 if interleaved else 0, out_at, out_stride, _raw_stream(dev)))
    return out


def causal_attention(q, k_cache, v_cache, new_start, length, max_new=None, max_len=None, cache_start=None, scale=0.0,
                     splits=0, out=None, workspace=None):
    """Causal attention of the new tokens over the cache (qlin_causal_attention in
    include/qlin_target.h).

    q: CUDA bf16 [rows, q heads, 128], rows may be apart; cache and batch as for
    ``norm_rope_append``.  max_new (default: the rows) and max_len (default: the
    cache's capacity) choose the kernel and its split: give 1 for single tokens, and
    chunks of prompts a call of their own.  ``workspace``
    (a CUDA tensor of at least the planned bytes) is allocated when needed and not
    given.  Returns ``out`` [rows, q heads, 128]; rows of no sequence are left as
    they are.
    """
    dev = _device()
    bf16 = _torch.bfloat16
    q_at = _address("q", q, bf16, dev)
    if q.dim() != 3:
        raise ValueError("q must have rank 3")
    rows, Hq, D = shape = q.shape
    q_stride = _row_stride("q", q, Hq)
    cache = _kv_cache(k_cache, v_cache, dev)
    batch = _batch(dev, rows, new_start, length, max_new, max_len, cache_start, k_cache)
    if workspace is None:
        size = batch.n_seq, rows, batch.max_new, batch.max_len, Hq, cache.heads, D, splits, dev
        need = _scratch_bytes.get(size)
        if need is None:
            need = ctypes.c_int64()
            _check(lib().qlin_causal_plan(batch, Hq, cache.heads, D, splits, None, ctypes.byref(need), None, 0))
            need = _remember(size, need.value)
        if need:
            workspace = _torch.empty(need, dtype=_torch.uint8, device=q.device)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the current CUDA device")
    if out is None:
        # of a contiguous tensor, empty_like costs half of empty
        out = _torch.empty_like(q) if q.is_contiguous() else _torch.empty(shape, dtype=bf16, device=q.device)
        out_at, out_stride = out.data_ptr(), Hq * D
    else:
        out_at = _address("out", out, bf16, dev)
        if out.shape != shape:
            raise ValueError(f"out must have shape {tuple(shape)}")
        out_stride = _row_stride("out", out, Hq)
    _check(lib().qlin_causal_attention(batch, cache, Hq, D, scale, splits, q_at, q_stride, out_at, out_stride,
                                       *_scratch(workspace), _raw_stream(dev)))
    return out


_scratch_bytes = {}                 # of a call's sizes


def _remember(size, need):
    if len(_scratch_bytes) >= 1024:
        _scratch_bytes.clear()
    _scratch_bytes[size] = need
    return need


def _scratch(workspace):
    """(address, bytes) of a workspace or None."""
    return (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())


def _logit_rows(name, t, n, rows, vocab):
    """Elements between the rows of [n, rows, vocab] logits, all rows at one distance."""
    if t.shape != (n, rows, vocab):
        raise ValueError(f"{name} must have shape {(n, rows, vocab)}")
    seq, row, one = t.stride()
    if rows == 1:
        row = seq
    if n * rows == 0:
        return vocab
    if (one != 1 and vocab > 1) or (n > 1 and seq != rows * row):
        raise ValueError(f"{name} must have contiguous rows at one distance")
    return row if n * rows > 1 else vocab


def verify_draft(target, drafted, uniform, draft=None, n_draft=None, temperature=None, accepted=None, tokens=None,
                 workspace=None):
    """Keep the accepted prefix of each sequence's drafted tokens and choose the next
    token (qlin_verify_draft in include/qlin_target.h).

    target: CUDA bf16 logits [n, drafts + 1, vocab]; drafted: int32 [n, drafts];
    uniform: float32 [n, drafts + 1] in [0, 1); draft: the drafter's bf16 logits [n,
    drafts, vocab], or None (its tokens had all its mass); n_draft: int32 [n] drafted
    tokens of each sequence, or None; temperature: float32 [n], or None (1).  Returns
    (accepted int32 [n], tokens int32 [n, drafts + 1], -1 behind the last).
    """
    dev = _device()
    bf16, i32, f32 = _torch.bfloat16, _torch.int32, _torch.float32
    target_at = _address("target", target, bf16, dev)
    if target.dim() != 3 or target.shape[1] == 0:
        raise ValueError("target must be [n, drafts + 1, vocab]")
    n, rows, vocab = target.shape
    target_stride = _logit_rows("target", target, n, rows, vocab)
    draft_at, draft_stride = None, vocab
    if draft is not None:
        draft_at = _address("draft", draft, bf16, dev)
        draft_stride = _logit_rows("draft", draft, n, rows - 1, vocab)
        if rows == 1:                                       # no drafted tokens, no rows
            draft_at = None
    if accepted is None:
        accepted = _torch.empty(n, dtype=i32, device=target.device)
    if tokens is None:
        tokens = _torch.empty((n, rows), dtype=i32, device=target.device)
    at = []
    for name, t, dtype, cols in (("drafted", drafted, i32, rows - 1), ("uniform", uniform, f32, rows), ("tokens", tokens, i32, rows)):
        at.append(_address(name, t, dtype, dev))
        if t.shape != (n, cols) or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous, of shape {(n, cols)}")
    if workspace is None:
        size = n, rows, vocab
        need = _scratch_bytes.get(size)
        if need is None:
            need = _remember(size, qlin_verify_plan(n, rows - 1, vocab))
        if need:
            workspace = _torch.empty(need, dtype=_torch.uint8, device=target.device)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the current CUDA device")
    _check(lib().qlin_verify_draft(n, rows - 1, vocab, target_at, target_stride, draft_at, draft_stride, at[0],
                                   _vector("n_draft", n_draft, i32, dev, n),
                                   _vector("temperature", temperature, f32, dev, n), at[1],
                                   _vector("accepted", accepted, i32, dev, n), at[2], *_scratch(workspace),
                                   _raw_stream(dev)))
    return accepted, tokens


def new_workspace(nbytes, device=None):
    """A zero-filled device workspace for forward_group (zero before first use)."""
    import torch
    return torch.zeros(max(int(nbytes), 16), dtype=torch.uint8, device=device or "cuda")


def forward_group(lins, x, outs=None, path=PATH_AUTO, split_k=0, workspace=None):
    """One launch over QLinear layers that share x (qlin_forward_group).
    ``workspace``: a zero-filled CUDA uint8 tensor (new_workspace), or None
    for plans without a K split.  Returns the list of outputs."""
    import torch
    K = lins[0].K
    for l in lins:
        if l.K != K:
            raise ValueError("the layers of a group must share K")
    x = lins[0]._check_x(x)
    M = x.shape[0]
    if outs is None:
        outs = [torch.empty((M, l.N), dtype=torch.bfloat16, device=x.device) for l in lins]
    else:
        for l, o in zip(lins, outs):
            _check_out(o, (M, l.N), x.device)
    wp, wb = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if workspace is not None else (None, 0)
    _check(qlin_forward_group([l.h for l in lins], path, split_k, M, x.data_ptr(), [o.data_ptr() for o in outs],
                              wp, wb, _stream()))
    return outs


def group_plan(lins, M, path=PATH_AUTO, split_k=0, ws_bytes=-1):
    """(workspace bytes, plan text) of forward_group over lins for M rows."""
    return qlin_group_plan([l.h for l in lins], path, split_k, M, ws_bytes)


class QLinear:
    """One W4A16 linear layer on the current GPU.

    ``packed``/``scales``/``zeros`` are host arrays or device tensors in the
    canonical layout (see include/qlin.h); ``zeros=None`` selects the
    symmetric format.
    """

    def __init__(self, packed, scales, zeros=None, group=128):
        if not hasattr(packed, "data_ptr"):
            packed = np.asarray(packed)
        self.N, K8 = packed.shape
        self.K = K8 * 8
        import torch
        self.device = torch.device("cuda", torch.cuda.current_device())
        if zeros is None:
            self.h = qlin_create_symmetric(self.K, self.N, group, packed, scales)
        else:
            self.h = qlin_create(self.K, self.N, group, packed, scales, zeros)

    def _check_x(self, x):
        import torch
        if x.dtype != torch.bfloat16 or x.device != self.device or x.dim() != 2 or x.shape[1] != self.K:
            raise ValueError(f"x must be a bf16 tensor of shape [M, {self.K}] on {self.device}")
        return x.contiguous()

    def forward(self, x, out=None, path=PATH_AUTO, split_k=0, workspace=None):
        """y = x . w^T.  With ``workspace`` (new_workspace) the call goes
        through qlin_forward_group and may use the plans that need it."""
        import torch
        if workspace is not None:
            return forward_group([self], x, None if out is None else [out], path, split_k, workspace)[0]
        x = self._check_x(x)
        M = x.shape[0]
        if out is None:
            y = torch.empty((M, self.N), dtype=torch.bfloat16, device=x.device)
        else:
            y = out
            _check_out(y, (M, self.N), x.device)
        _check(qlin_forward_path(self.h, path, split_k, M, x.data_ptr(), y.data_ptr(), _stream()))
        return y

    __call__ = forward

    def workspace_bytes(self):
        """Bytes of the handle's own workspace."""
        return qlin_workspace_bytes(self.h)

    def plan(self, M, path=PATH_AUTO, split_k=0):
        return qlin_plan(self.h, path, split_k, M)

    def unpack_codes(self):
        import torch
        q = torch.empty((self.N, self.K), dtype=torch.uint8, device="cuda")
        _check(qlin_unpack_codes(self.h, q.data_ptr(), _stream()))
        return q

    def dequantize(self, routine=0):
        import torch
        w = torch.empty((self.N, self.K), dtype=torch.bfloat16, device="cuda")
        _check(qlin_dequantize(self.h, routine, w.data_ptr(), _stream()))
        return w

    def close(self):
        if getattr(self, "h", None):
            qlin_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

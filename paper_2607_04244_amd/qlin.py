"""Python binding of ``libqlin.so`` (argument marshalling only).

The functions mirror the C ABI in ``include/qlin.h`` one to one; ``QLinear``
wraps a handle for torch callers.  torch supplies device memory and the
current stream; every step of the computation runs in the HIP kernels.  The
module raises if the library has not been built - there is no fallback.
"""

import ctypes
import os

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


class KVCache(ctypes.Structure):
    """struct qlin_kv_cache (include/qlin_target.h); strides in elements."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("heads", ctypes.c_int64), ("slots", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("seq_slots", ctypes.c_int64)]


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


def _need(name, t, dtype, device, shape=None, rank=None):
    """Raise unless t is a tensor of this type, device and shape (None entries: any size)."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be a {dtype} tensor on {device}")
    if rank is not None and t.dim() != rank:
        raise ValueError(f"{name} must have rank {rank}")
    if shape is not None and (t.dim() != len(shape) or any(w is not None and n != w for n, w in zip(t.shape, shape))):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")


def _current(name, t):
    """The device of a tensor, which has to be the current one (the stream's)."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} must be a tensor on the current CUDA device")
    return t.device


def _ptr(t):
    return None if t is None else t.data_ptr()


def _kv_cache(k_cache, v_cache, device, cache_start):
    """KVCache of [sequences, heads, capacity, 128] or packed [tokens, heads, 128] tensors."""
    import torch
    for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
        _need(name, t, torch.bfloat16, device)
    if k_cache.shape != v_cache.shape or k_cache.stride() != v_cache.stride():
        raise ValueError("k_cache and v_cache must have the same shape and strides")
    if k_cache.dim() not in (3, 4) or k_cache.shape[-1] != 128 or k_cache.stride(-1) != 1 or k_cache.numel() == 0:
        raise ValueError("the cache must be [sequences, heads, capacity, 128] or [tokens, heads, 128], rows contiguous")
    if k_cache.dim() == 3:
        slots, heads, _ = k_cache.shape
        token, head, _ = k_cache.stride()
        return KVCache(k_cache.data_ptr(), v_cache.data_ptr(), heads, slots, token, head, 0)
    n, heads, capacity, _ = k_cache.shape
    seq, head, token, _ = k_cache.stride()
    if n == 1:
        seq = 0
    if token <= 0 or seq % token:
        raise ValueError("the cache's sequences must lie whole tokens apart")
    seq_slots = seq // token
    return KVCache(k_cache.data_ptr(), v_cache.data_ptr(), heads, (n - 1) * seq_slots + capacity, token, head, seq_slots)


def _batch(device, rows, new_start, length, max_new, max_len, cache_start, k_cache):
    import torch
    _need("length", length, torch.int32, device, rank=1)
    n = length.shape[0]
    _need("new_start", new_start, torch.int32, device, (n + 1,))
    if cache_start is not None:
        _need("cache_start", cache_start, torch.int64, device, (n,))
    for name, t in (("length", length), ("new_start", new_start), ("cache_start", cache_start)):
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    if cache_start is None and n > 1 and (k_cache.dim() == 3 or k_cache.shape[0] < n):
        raise ValueError("several sequences need cache_start or a cache of as many sequences")
    if max_len is None:
        max_len = k_cache.shape[2] if k_cache.dim() == 4 else k_cache.shape[0]
    return Batch(n, rows, rows if max_new is None else min(max_new, rows), max_len, new_start.data_ptr(),
                 length.data_ptr(), _ptr(cache_start))


def _check_out_rows(name, t, shape, device):
    """An output [rows, heads, 128] whose rows may be apart."""
    import torch
    _need(name, t, torch.bfloat16, device, shape)
    if t.stride(2) != 1 or (t.shape[1] > 1 and t.stride(1) != 128):
        raise ValueError(f"{name}: the heads of a row must be contiguous")


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
    import torch
    device = _current("q", q)
    for name, t in (("q", q), ("k", k), ("v", v)):
        _need(name, t, torch.bfloat16, device, rank=2)
        if t.shape[1] == 0 or t.shape[1] % 128 or t.stride(1) != 1 or t.shape[0] != q.shape[0]:
            raise ValueError(f"{name} must be [rows, heads * 128] with contiguous rows")
    cache = _kv_cache(k_cache, v_cache, device, cache_start)
    rows, Hq = q.shape[0], q.shape[1] // 128
    if k.shape[1] != cache.heads * 128 or v.shape[1] != cache.heads * 128:
        raise ValueError(f"k and v must have the cache's {cache.heads} heads")
    batch = _batch(device, rows, new_start, length, max_new, max_len, cache_start, k_cache)
    for name, t in (("q_norm", q_norm), ("k_norm", k_norm)):
        if t is not None:
            _need(name, t, torch.bfloat16, device, (128,))
    if inv_freq is not None:
        _need("inv_freq", inv_freq, torch.float64, device, rank=1)
    for name, t in (("q_norm", q_norm), ("k_norm", k_norm), ("inv_freq", inv_freq)):
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    if out is None:
        out = torch.empty((rows, Hq, 128), dtype=torch.bfloat16, device=device)
    else:
        _check_out_rows("out", out, (rows, Hq, 128), device)
    stride = [t.stride(0) if rows > 1 else t.shape[1] for t in (q, k, v)]
    _check(qlin_norm_rope_append(batch, cache, Hq, 128, q.data_ptr(), stride[0], k.data_ptr(), stride[1], v.data_ptr(),
                                 stride[2], _ptr(q_norm), _ptr(k_norm), eps, _ptr(inv_freq),
                                 0 if inv_freq is None else 2 * inv_freq.shape[0], int(interleaved), out.data_ptr(),
                                 out.stride(0) if rows > 1 else Hq * 128, _stream()))
    return out


def causal_attention(q, k_cache, v_cache, new_start, length, max_new=None, max_len=None, cache_start=None, scale=0.0,
                     splits=0, out=None, workspace=None):
    """Causal attention of the new tokens over the cache (qlin_causal_attention in
    include/qlin_target.h).

    q: CUDA bf16 [rows, q heads, 128], rows may be apart; cache and batch as for
    ``norm_rope_append``.  max_new and max_len size the work split.  ``workspace``
    (a CUDA tensor of at least the planned bytes) is allocated when needed and not
    given.  Returns ``out`` [rows, q heads, 128]; rows of no sequence are left as
    they are.
    """
    import torch
    device = _current("q", q)
    _need("q", q, torch.bfloat16, device, rank=3)
    rows, Hq, D = q.shape
    _check_out_rows("q", q, (rows, Hq, D), device)
    cache = _kv_cache(k_cache, v_cache, device, cache_start)
    batch = _batch(device, rows, new_start, length, max_new, max_len, cache_start, k_cache)
    if workspace is None:
        _, nbytes, _ = qlin_causal_plan(batch, Hq, cache.heads, D, splits)
        if nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    elif workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    if out is None:
        out = torch.empty((rows, Hq, D), dtype=torch.bfloat16, device=device)
    else:
        _check_out_rows("out", out, (rows, Hq, D), device)
    _check(qlin_causal_attention(batch, cache, Hq, D, scale, splits, q.data_ptr(), q.stride(0) if rows > 1 else Hq * D,
                                 out.data_ptr(), out.stride(0) if rows > 1 else Hq * D, _ptr(workspace),
                                 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))
    return out


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
    import torch
    device = _current("target", target)
    _need("target", target, torch.bfloat16, device, rank=3)
    n, rows, vocab = target.shape
    _need("drafted", drafted, torch.int32, device, (n, rows - 1))
    _need("uniform", uniform, torch.float32, device, (n, rows))
    if draft is not None:
        _need("draft", draft, torch.bfloat16, device, (n, rows - 1, vocab))
        draft = draft if rows > 1 else None                 # no drafted tokens, no rows
    if n_draft is not None:
        _need("n_draft", n_draft, torch.int32, device, (n,))
    if temperature is not None:
        _need("temperature", temperature, torch.float32, device, (n,))
    strides = []
    for name, t in (("target", target), ("draft", draft)):
        if t is None or t.shape[0] * t.shape[1] <= 1:
            row = vocab
        else:
            row = t.stride(1) if t.shape[1] > 1 else t.stride(0)
        if t is not None and (t.stride(2) != 1 or (t.shape[0] > 1 and t.stride(0) != t.shape[1] * row)):
            raise ValueError(f"{name} must have contiguous rows at one distance")
        strides.append(row)
    if accepted is None:
        accepted = torch.empty(n, dtype=torch.int32, device=device)
    if tokens is None:
        tokens = torch.empty((n, rows), dtype=torch.int32, device=device)
    _need("accepted", accepted, torch.int32, device, (n,))
    _need("tokens", tokens, torch.int32, device, (n, rows))
    for name, t in (("drafted", drafted), ("uniform", uniform), ("n_draft", n_draft), ("temperature", temperature),
                    ("accepted", accepted), ("tokens", tokens), ("workspace", workspace)):
        if t is not None and (t.device != device or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous tensor on {device}")
    if workspace is None:
        nbytes = qlin_verify_plan(n, rows - 1, vocab)
        if nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    _check(qlin_verify_draft(n, rows - 1, vocab, target.data_ptr(), strides[0], _ptr(draft), strides[1],
                             drafted.data_ptr(), _ptr(n_draft), _ptr(temperature), uniform.data_ptr(),
                             accepted.data_ptr(), tokens.data_ptr(), _ptr(workspace),
                             0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))
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

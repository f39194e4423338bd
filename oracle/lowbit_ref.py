"""CPU oracle of a layer's operators in fewer bits: norms around a block, 8-bit tokens and
their linear, rows of a 4-bit key/value cache.

TEST INFRASTRUCTURE ONLY.  Only ``tests/`` may import it.  It shares no code with
``paper_2607_04244_amd`` and imports nothing from it.

Definitions:

* Block norm: h = bf16(residual + scale * norm(y, post) * gate), out = norm(h, pre), with
  norm(x, w) = x / sqrt(mean(x^2) + eps) * w.
* Tokens: scale = max |v| / 127 in binary32, codes = v / scale rounded to nearest, ties to
  even; v = x or silu(a) b of the two halves.
* 8-bit linear: bf16(binary32(sum) * (x_scale * w_scale)).
* 4-bit rows of 128 bf16 values: offset = min, step = bf16((max - min) / 15) in binary32,
  codes = (x - offset) / step rounded to nearest, ties to even, at most 15.

Plain numpy, float64 unless a definition names binary32.  Pinned by
``tests/test_oracle_lowbit.py``.
"""

import numpy as np

HEAD = 128
F32 = np.float32


def to_bf16(x):
    """float64 -> binary32 -> bf16, to nearest with ties to even; as float64 (NaN stays NaN)."""
    with np.errstate(over="ignore"):
        f = np.asarray(x, dtype=np.float64).astype(F32)
    u = f.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    return np.where(np.isnan(f), np.nan, r.view(F32).astype(np.float64))


def norm(x, w, eps):
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * w


def block_norm(y, residual, post=None, gate=None, sigmoid=False, scale=1.0, eps=1e-6):
    """(h before its rounding, the added part) of float64 rows."""
    t = y if post is None else norm(y, post, eps)
    if gate is not None:
        t = t * (1.0 / (1.0 + np.exp(-gate)) if sigmoid else gate)
    return residual + scale * t, scale * t


def silu_product(x):
    a, b = np.split(x, 2, axis=-1)
    return a / (1.0 + np.exp(-a)) * b


def quantize_tokens(v):
    """(codes int8, scale binary32) of rows of binary32 values."""
    v = np.asarray(v, dtype=F32)
    peak = np.max(np.abs(v), axis=-1)                        # NaN if any is
    scale = (peak / F32(127)).astype(F32)
    bad, zero = ~np.isfinite(peak), peak < 2.0 ** -100
    with np.errstate(all="ignore"):
        codes = np.rint((v / scale[..., None]).astype(F32))
    codes[bad | zero] = 0
    return codes.astype(np.int8), np.where(bad, F32(np.nan), np.where(zero, F32(0), scale)).astype(F32)


def linear_i8(x, x_scale, w, w_scale):
    """float64 values of the bf16 outputs."""
    total = x.astype(np.int64) @ w.astype(np.int64).T
    assert np.abs(total).max(initial=0) < 2 ** 31
    with np.errstate(over="ignore"):
        return to_bf16(total.astype(F32) * (x_scale.astype(F32)[:, None] * w_scale.astype(F32)[None]))


def lay_on_grid(x):
    """(codes [..., 128], step, offset) of float64 rows of bf16 values."""
    x = np.asarray(x, dtype=np.float64)
    low, high = x.min(axis=-1), x.max(axis=-1)               # NaN if any is
    with np.errstate(all="ignore"):
        span = (high.astype(F32) - low.astype(F32)).astype(F32)
        step = to_bf16((span / F32(15)).astype(F32))
        step = np.where(step < 2.0 ** -126, 0.0, step)
        q = ((x - low[..., None]).astype(F32) / step.astype(F32)[..., None]).astype(F32)
    codes = np.where(step[..., None] > 0, np.minimum(np.rint(q), 15), 0)
    bad = ~np.isfinite(span)
    codes[bad] = 0
    return codes.astype(np.int64), np.where(bad, np.nan, step), np.where(bad, np.nan, low)


def pack_codes(codes):
    """[..., 128] codes -> [..., 16] uint32 words, the first code in the lowest bits."""
    c = codes.reshape(*codes.shape[:-1], 16, 8).astype(np.uint64)
    return np.sum(c << (4 * np.arange(8, dtype=np.uint64)), axis=-1).astype(np.uint32)


def unpack_codes(words):
    w = words.astype(np.uint32)[..., None] >> (4 * np.arange(8, dtype=np.uint32))
    return (w & 15).reshape(*words.shape[:-1], HEAD).astype(np.int64)


def row_values(words, step, offset):
    """float64 values of rows of words."""
    return step[..., None] * unpack_codes(words) + offset[..., None]

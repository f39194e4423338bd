"""The oracle of the operators in fewer bits, pinned by closed forms and plain loops (CPU)."""

import math

import numpy as np
import torch

from oracle import lowbit_ref as ref


def bf16(values):
    return torch.tensor(values, dtype=torch.float32).to(torch.bfloat16).double().numpy()


def test_bf16_rounding_is_that_of_torch():
    x = np.concatenate([np.random.default_rng(0).standard_normal(5000) * 10.0 ** np.random.default_rng(1).integers(-30, 30, 5000),
                        [0.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -1 - 2.0 ** -8, 3.4e38, 2.0 ** -130]])
    assert np.array_equal(ref.to_bf16(x), torch.tensor(x).float().to(torch.bfloat16).double().numpy())
    assert np.isnan(ref.to_bf16(np.nan))


def test_block_norm_of_known_rows():
    y, r = np.array([[3.0, 4.0]]), np.array([[10.0, 20.0]])
    h, t = ref.block_norm(y, r, post=np.array([1.0, 2.0]), gate=np.array([[0.0, 0.0]]), sigmoid=True, scale=4.0, eps=0.0)
    rms = math.sqrt(12.5)
    assert np.allclose(t, [[4 * 0.5 * 3 / rms, 4 * 0.5 * 2 * 4 / rms]]) and np.allclose(h, r + t)
    assert np.array_equal(ref.block_norm(y, r)[0], r + y)


def test_tokens_of_known_rows():
    codes, scale = ref.quantize_tokens(np.array([[127.0, -127.0, 0.5, 1.5, -2.5], [0.0] * 5, [1.0, 2.0, np.inf, 0.0, 0.0]]))
    assert codes[0].tolist() == [127, -127, 0, 2, -2] and scale[0] == 1.0           # ties to even
    assert codes[1].tolist() == [0] * 5 and scale[1] == 0.0
    assert codes[2].tolist() == [0] * 5 and np.isnan(scale[2])


def test_silu_product_of_known_values():
    assert np.allclose(ref.silu_product(np.array([[0.0, 2.0, 5.0, 3.0]])), [[0.0, 3 * 2 / (1 + math.exp(-2))]])


def test_linear_by_plain_loops():
    g = np.random.default_rng(2)
    x, w = g.integers(-127, 128, (3, 32)).astype(np.int8), g.integers(-127, 128, (5, 32)).astype(np.int8)
    sx, sw = g.random(3).astype(np.float32), g.random(5).astype(np.float32)
    y = ref.linear_i8(x, sx, w, sw)
    for m in range(3):
        for n in range(5):
            total = sum(int(x[m, k]) * int(w[n, k]) for k in range(32))
            want = np.float32(np.float32(total) * np.float32(sx[m] * sw[n]))
            assert y[m, n] == float(torch.tensor(want).to(torch.bfloat16))


def test_grid_of_known_rows():
    x = np.zeros((3, 128))
    x[0] = np.arange(128) % 16                     # the grid itself
    x[1] = 7.0                                     # one value
    x[2, :] = bf16([0.0] * 128)
    x[2, 0], x[2, 1], x[2, 2] = 15.0, 0.5, 1.5     # ties to even
    codes, step, offset = ref.lay_on_grid(x)
    assert step.tolist() == [1.0, 0.0, 1.0] and offset.tolist() == [0.0, 7.0, 0.0]
    assert codes[0].tolist() == list(np.arange(128) % 16) and not codes[1].any() and codes[2, :4].tolist() == [15, 0, 2, 0]
    words = ref.pack_codes(codes)
    assert words[0, 0] == 0x76543210 and words[0, 1] == 0xFEDCBA98
    assert np.array_equal(ref.unpack_codes(words), codes)
    assert np.array_equal(ref.row_values(words, step, offset)[0], x[0])


def test_grid_is_within_half_a_step():
    g = np.random.default_rng(3)
    x = ref.to_bf16(g.standard_normal((200, 128)) * np.exp(g.standard_normal((200, 1)) * 4))
    codes, step, offset = ref.lay_on_grid(x)
    values = ref.row_values(ref.pack_codes(codes), step, offset)
    # half a step, and the top value what a step rounded down (2^-8 of it, 15 times) misses
    assert np.all(np.abs(values - x) <= step[:, None] * (0.5 + 15 * 2.0 ** -8))
    assert codes.min() == 0 and codes.max() == 15


def test_grid_of_rows_without_numbers():
    x = np.ones((3, 128))
    x[0, 5], x[1, 6] = np.inf, np.nan
    x[2, 0], x[2, 1] = 3e38, -3e38
    codes, step, offset = ref.lay_on_grid(x)
    assert not codes.any() and np.isnan(step).all() and np.isnan(offset).all()

"""Pins of the oracle of the target's operators (CPU): closed forms, loops over tiny
inputs, and the law the verification keeps (its tokens follow the target)."""

import math

import numpy as np

from oracle import target_ref as ref


def test_norm_of_a_constant_row_is_the_weight():
    x = np.full((1, 128), -3.0)
    w = np.linspace(0.5, 2.0, 128)
    assert np.allclose(ref.norm(x, w, 0.0), -w)
    assert np.allclose(ref.norm(x, w, 27.0), -w * 3.0 / 6.0)         # sqrt(9 + 27) = 6
    assert ref.norm(x, None, 1.0) is x


def test_rotation_pairs_and_turns():
    x = np.zeros((1, 128))
    x[0, 1] = 1.0
    freq = np.full(16, math.pi / 2)                                  # a quarter turn a position
    y = ref.rotate(x, 1, freq, False)
    assert abs(y[0, 17] - 1) < 1e-15 and abs(y[0, 1]) < 1e-15        # (1, 1 + 16)
    y = ref.rotate(x, 1, freq, True)
    assert abs(y[0, 0] + 1) < 1e-15                                  # (0, 1): second of its pair
    assert np.allclose(ref.rotate(x, 4, freq, False), x, atol=1e-14)
    z = np.random.default_rng(0).standard_normal((3, 128))
    assert np.allclose(np.linalg.norm(ref.rotate(z, 7, freq, True), axis=1), np.linalg.norm(z, axis=1))
    assert np.array_equal(ref.rotate(z, 7, freq, False)[:, 32:], z[:, 32:])


def test_rotated_products_depend_on_the_distance_alone():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((1, 128)), rng.standard_normal((1, 128))
    freq = 1e4 ** (-np.arange(64) / 64)
    for il in (False, True):
        a = (ref.rotate(q, 9, freq, il) * ref.rotate(k, 5, freq, il)).sum()
        b = (ref.rotate(q, 1009, freq, il) * ref.rotate(k, 1005, freq, il)).sum()
        assert abs(a - b) < 1e-9


def test_positions():
    assert ref.positions([2, 0, 1], [5, 9, 1]) == [(0, 3), (0, 4), (2, 0)]


def test_attention_closed_forms():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((7, 2, 128)), rng.standard_normal((7, 2, 128))
    out, _ = ref.causal_attention(np.zeros((3, 4, 128)), k, v, 1.0)
    for i in range(3):
        for h in range(4):
            assert np.allclose(out[i, h], v[:5 + i, h // 2].mean(axis=0))    # equal weights over what is seen
    out, _ = ref.causal_attention(np.zeros((9, 2, 128)), k, v, 1.0)         # more new tokens than cached
    assert np.all(out[:2] == 0) and np.allclose(out[2, 0], v[0, 0])
    q = 100.0 * k[3:4, :1].repeat(2, 1)
    out, _ = ref.causal_attention(q, k, v, 1.0)
    assert np.allclose(out[0, 0], v[3, 0], atol=1e-9)                        # one dominant key


def test_attention_loops():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((2, 2, 128)), rng.standard_normal((4, 1, 128)), rng.standard_normal((4, 1, 128))
    out, spread = ref.causal_attention(q, k, v, 0.1)
    for i in range(2):
        for h in range(2):
            e = [math.exp(0.1 * math.fsum(q[i, h] * k[j, 0])) for j in range(3 + i)]
            for d in (0, 77):
                assert abs(out[i, h, d] - math.fsum(e[j] * v[j, 0, d] for j in range(3 + i)) / math.fsum(e)) < 1e-12
                assert abs(spread[i, h, d] - math.fsum(e[j] * abs(v[j, 0, d]) for j in range(3 + i)) / math.fsum(e)) < 1e-12


def test_verify_greedy_and_masks():
    t = np.array([[0.0, 2.0, 2.0], [5.0, 1.0, 0.0], [0.0, 0.0, 1.0]])
    assert ref.verify(t, None, [1, 0], [0.9, 0.9, 0.5], 0.0) == (2, 2)
    assert ref.verify(t, None, [2, 0], [0.9, 0.9, 0.5], 0.0) == (0, 1)       # ties: the lowest index
    t[0] = [-np.inf, np.nan, -np.inf]
    assert ref.verify(t, None, [1, 0], [0.0, 0.0, 0.5], 1.0) == (0, -1)      # nothing left
    assert ref.verify(t[1:2], None, [], [0.0], 0.0) == (0, 0)                # plain sampling
    assert ref.verify(t[1:], None, [7], [0.0, 0.0], 1.0)[0] == 0             # outside the vocabulary
    assert ref._distribution(np.array([np.inf, 1.0, np.inf]), 1.0).tolist() == [0.5, 0.0, 0.5]


def test_verify_draws_from_the_target():
    """The first token's law over random draws equals the target's, with a drafter that
    samples its own law and with one that always proposes its best token."""
    rng = np.random.default_rng(4)
    V, N = 5, 40000
    t, d = rng.standard_normal((2, V)), rng.standard_normal((1, V))
    p = np.exp(t[0]) / np.exp(t[0]).sum()
    q = np.exp(d[0]) / np.exp(d[0]).sum()
    for with_draft in (True, False):
        counts = np.zeros(V)
        for _ in range(N):
            x = int(rng.choice(V, p=q)) if with_draft else int(d[0].argmax())
            a, nxt = ref.verify(t, d if with_draft else None, [x], rng.random(2), 1.0)
            counts[x if a else nxt] += 1
        # 5 standard deviations of a binomial share
        assert np.all(np.abs(counts / N - p) < 5 * np.sqrt(p * (1 - p) / N))

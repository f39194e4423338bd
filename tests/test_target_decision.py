"""GPU tests of qlin_verify_draft at the ends of its range, against the float64 oracle
(whole numbers: equal)."""

import numpy as np
import pytest
import torch

from test_target import check_verify, rand, verify_case

pytestmark = pytest.mark.gpu

MOST = float(torch.finfo(torch.bfloat16).max)


def sampled(target, u, T):
    """Plain sampling of every row: [n, 1, V], one uniform number and temperature each."""
    n = target.shape[0]
    return check_verify(target, None, [[]] * n, [[x] for x in u], T=T)


# ---------------------------------------------------------------- large logits over a temperature


@pytest.mark.parametrize("V", [4, 4099])
@pytest.mark.parametrize("top", [17.25, -17.25, 1e-3, 1e20, -1e20, MOST, -MOST])
def test_exponents_of_large_logits_over_small_temperatures(top, V):
    """The largest logit has the weight 1 however large |logit| / T is, and its equals too."""
    temperatures = [1e-45, 1e-38, 1e-30, 1e-20, 1e-10, 1e-6, 0.3, 0.5, 0.6, 0.7, 0.8, 1.0, 1.7, 1e20, float("inf")]
    low = -2.0 if abs(top) < 1e10 else -MOST
    values = [low, 0.25 * top if top > 0 else 2 * top if top > -1e30 else low, top, low]
    t = torch.full((len(temperatures), 1, V), low, dtype=torch.bfloat16)
    t[:, :, :4] = torch.tensor(values, dtype=torch.bfloat16)
    for u in (0.0, 0.3, 0.99):
        sampled(t, [u] * len(temperatures), temperatures)
    t[:, :, V - 1] = t[:, :, 2]                                          # a tie, in another chunk if there are two
    for u in (0.0, 0.3, 0.7, 0.99):
        sampled(t, [u] * len(temperatures), temperatures)


@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("mask", [1e20, -1e20, MOST, -MOST])
def test_decisions_with_forced_and_masked_logits(mask, with_draft):
    """Logits forced up or masked by finite numbers, in the target, the draft or both."""
    target, draft, drafted, u = verify_case(6, 3, 9001, 4, with_draft=with_draft)
    force = torch.zeros(9001, dtype=torch.bool)
    force[[5, 700, 8999] if mask > 0 else slice(0, 9001, 2)] = True
    target[:3, :, force] = mask
    if with_draft:
        draft[1:4, :, force] = mask
    for T in ([1.0] * 6, [0.5, 0.6, 0.7, 0.8, 0.9, 1.3], [1e-20, 1e-12, 1e-8, 1e-5, 1e-20, 0.0]):
        check_verify(target, draft, drafted, u, T=T)
    drafted = [[5, 700, 5]] * 6
    check_verify(target, draft, drafted, u, T=[0.8, 1.0, 0.7, 0.6, 1e-15, 1e-30])


# ---------------------------------------------------------------- equal rows


@pytest.mark.parametrize("V,stride", [(64, None), (4097, None), (50257, None), (9000, 9001), (20011, 20013)])
def test_equal_rows_leave_the_target_when_a_token_is_refused(V, stride):
    """Where target and draft agree, a token of probability 0 is refused and nothing is left
    of P - Q: the next token comes from P, at any distance of the rows from 16 bytes."""
    n, drafts = 6, 3
    target = rand(V, (n, drafts + 1, V), 2.0)
    target[:, :, 7] = float("-inf")
    draft = target[:, :drafts].clone()
    drafted = [[-1, 2, 3], [7, 2, 3], [V, 1, 1], [2, -5, 1], [3, 4, 7], [1, 7, 7]]
    T = [1.0, 0.7, 1.3, 1.0, 0.9, 2.0]
    for u in (0.0, 0.1, 0.37, 0.5, 0.83, 0.999):
        acc = check_verify(target, draft, drafted, [[0.5] * drafts + [u]] * n, T=T, stride=stride)
        assert acc == [0, 0, 0, 1, 2, 1]


def test_nearly_equal_rows_are_told_apart():
    """One logit that differs by a step of bf16: the rest of P - Q is that token alone, or all
    the others."""
    V = 3000
    target = rand(3, (2, 2, V), 1.0)
    draft = target[:, :1].clone()
    draft[0, 0, 1234] = 0.5
    draft[1, 0, 1234] = 0.5
    target[0, 0, 1234] = 0.50390625                                      # more probable: the only token of the rest
    target[1, 0, 1234] = 0.498046875                                     # less: all others share the rest
    for u in (0.0, 0.2, 0.6, 0.97):
        check_verify(target, draft, [[-1], [-1]], [[0.5, u]] * 2)


# ---------------------------------------------------------------- weights at the end of the range


@pytest.mark.parametrize("low", [-600.0, -744.0, -740.0, -710.0, -1000.0, -1e4, -1e9])
@pytest.mark.parametrize("V", [8192, 8189, 12288])
def test_chunks_of_vanishing_weight_hold_no_token(low, V):
    """u = 0 draws the first token of any weight: not one of a chunk whose weights are no
    numbers any more, relative to the largest (e^-600 still is one)."""
    t = torch.full((1, 2, V), low, dtype=torch.bfloat16)
    t[:, :, 4096:] = 0.0
    for u in (0.0, 1e-30, 0.5):
        acc, tok = decide(t, None, [[-1]], [[0.5, u]])
        assert acc == [0] and 0 <= tok[0][0] < V
        if low > -650.0 and u == 0.0:
            assert tok[0][0] == 0
        elif low < -740.0 or u > 0.0:
            assert tok[0][0] >= 4096 - (8 if u > 0.0 else 0)
    if low < -740.0 or low > -650.0:
        check_verify(t, None, [[-1]], [[0.5, 0.0]])
        check_verify(t, None, [[-1]], [[0.5, 0.9]])


def test_a_refused_token_that_had_almost_all_of_its_chunk():
    """The refused token held all but 2^-50 of its chunk, which itself is e^-600 of the row."""
    V = 8192
    t = torch.full((1, 2, V), float("-inf"), dtype=torch.bfloat16)
    t[:, :, 5] = -600.0
    t[:, :, 9] = -636.0
    t[:, :, 5000] = 0.0
    check_verify(t, None, [[5]], [[0.5, 0.0]])
    check_verify(t, None, [[5]], [[0.5, 0.5]])


def decide(target, draft, drafted, u, T=None):
    from paper_2607_04244_amd import qlin
    n, r, _ = target.shape
    f32 = lambda x: torch.tensor(x, dtype=torch.float32, device="cuda")
    acc, tok = qlin.verify_draft(target.cuda(), torch.tensor(drafted, dtype=torch.int32, device="cuda").view(n, r - 1), f32(u).view(n, r),
                                 draft=None if draft is None else draft.cuda(), temperature=None if T is None else f32(T))
    torch.cuda.synchronize()
    return acc.tolist(), tok.tolist()


@pytest.mark.parametrize("seed", range(40))
def test_every_token_is_one_of_the_vocabulary(seed):
    """Rows of wild values: the next token always has a number of the vocabulary and a logit
    that is not masked, and equals the oracle's where that is settled."""
    rng = np.random.default_rng(seed)
    V, n, drafts = int(rng.choice([3, 100, 4096, 4100, 13001])), 4, 2
    pool = [0.0, 1.0, -1.0, 30.0, -700.0, -745.0, 1e3, -1e4, 1e20, -1e20, MOST, -MOST, float("-inf"), 1e-30]
    pick = lambda *shape: torch.tensor(np.asarray(pool)[rng.integers(0, len(pool), shape) if seed % 2 else
                                                        rng.choice(rng.integers(0, len(pool), 3), shape)]).to(torch.bfloat16)
    target, draft = pick(n, drafts + 1, V), pick(n, drafts, V) if seed % 3 else None
    target[:, :, int(rng.integers(V))] = 2.0
    drafted = rng.integers(-1, V, (n, drafts)).tolist()
    u = rng.choice([0.0, 1e-20, 0.25, 0.5, 0.99999], (n, drafts + 1)).tolist()
    T = rng.choice([1e-30, 1e-3, 0.5, 1.0, 2.0, 1e10], n).tolist()
    acc, tok = decide(target, draft, drafted, u, T)
    for b in range(n):
        assert 0 <= acc[b] <= drafts
        nxt = tok[b][acc[b]]
        assert 0 <= nxt < V and float(target[b, acc[b], nxt]) > float("-inf"), (b, acc[b], nxt)


@pytest.mark.parametrize("low", [-709.0, -716.0, -720.0, -732.0, -740.0])
def test_equal_rows_with_tokens_of_vanishing_weight(low):
    """Probabilities that are subnormal numbers differ by their rounding too: no part of the rest."""
    V, n = 700, 6
    target = rand(5, (n, 2, V), 1.0)
    target[:, :, 3:400] = (low + 8 * torch.rand((n, 2, 397), generator=torch.Generator().manual_seed(6))).to(torch.bfloat16)
    draft = target[:, :1].clone()
    for u in (0.0, 0.3, 0.9):
        acc, tok = decide(target, draft, [[-1]] * n, [[0.5, u]] * n, T=[1.0, 0.9, 1.1, 1.0, 0.95, 1.05])
        for b in range(n):
            assert acc[b] == 0 and 0 <= tok[b][0] < V
            assert u == 0.0 or not 3 <= tok[b][0] < 400                  # from P, where those have no weight to speak of
        if u > 0.0:
            check_verify(target, draft, [[-1]] * n, [[0.5, u]] * n, T=[1.0, 0.9, 1.1, 1.0, 0.95, 1.05])

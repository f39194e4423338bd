"""The causal attention over the 4-bit cache against float64, in the 2-norm (GPU).

Element by element, the attention's worst case says little: all errors of one sign, on the
largest of the values.  Here the relative 2-norm error of outputs stays below what independent
roundings, uniform within half a step, add up to, so an operand of fewer bits, a wrong power of
two of a head or row, or a lost key shows.  With p the weights, v the values, t an output:
* its own rounding to bf16: r, the error of the rounded float64 result, computed as it is;
* an operand in f16 is off by at most 2^-12, in the mean square by a = 2^-12 / sqrt(3).  Queries are
  bf16 and exact there.  The direct forms round p s (v = s c + o): a sqrt(sum_j p_j^2 s_j^2 c_j^2).  The
  forms that unpack round k, v and p: a score by a scale sqrt(sum_d q_d^2 k_d^2), an output by
  a sqrt(2) sqrt(sum_j p_j^2 v_j^2); a score off by e_j moves it by sum_j p_j e_j (v_j - t).
A rounding of p s is the same in all 128 dimensions, which leaves few independent ones over few keys:
the operands' part counts sqrt(2) times.  The whole 1.1 times, as at least 1000 outputs are
compared.  fp32 sums and exponentials are 2^-17 and less.  Operands of bf16 have 16 times the part of
f16: that this does not fit the bound is asserted, from the same numbers.
"""

import numpy as np
import pytest
import torch

from paper_2607_04244_amd import qlin

from test_kv4 import HEAD, UNPACKED, Cache, f64, i32, plan_text, rand, starts

A2 = 2.0 ** -24 / 3                      # mean square of an f16 operand's rounding


def errors(q, c, b, Hkv, scale, unpacked):
    """A sequence's new tokens: (float64 result, its squared error from the bf16 rounding, from the
    operands), each [n, Hq, 128]."""
    parts = [tuple(torch.from_numpy(np.ascontiguousarray(t)) for t in c.values(w, b)) for w in (0, 1)]
    n, Hq, _ = q.shape
    G, L = Hq // Hkv, c.length[b]
    q = torch.from_numpy(q)
    hidden = torch.arange(L)[None] > (L - n + torch.arange(n))[:, None]
    want, operands = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for h in range(Hq):
        (k, _, _), (v, _, vo) = (tuple(t[:, h // G] for t in part) for part in parts)
        p = torch.softmax((q[:, h] @ k.T * scale).masked_fill(hidden, -float("inf")), 1)
        t = p @ v
        if unpacked:
            moved = p.square() * (q[:, h].square() @ k.square().T * scale ** 2)
            operands[:, h] = moved @ v.square() - 2 * t * (moved @ v) + t.square() * moved.sum(1, keepdim=True) + 2 * (p.square() @ v.square())
        else:
            operands[:, h] = p.square() @ (v - vo[:, None]).square()
        want[:, h] = t
    own = (want.float().to(torch.bfloat16).double() - want).square()
    return want, own, A2 * operands.clamp_min(0)


def within(have, want, own, operands, what):
    """The relative errors over whatever is left of the arrays, all of them."""
    size = want.square().sum()
    error = float(((have - want).square().sum() / size).sqrt())
    own, operands = float(own.sum() / size), float(operands.sum() / size)
    bound = 1.1 * (own + 2 * operands) ** 0.5
    assert have.numel() >= 1000 and bound < 0.004
    assert bound < (own + 256 * operands) ** 0.5, f"{what}: bf16 operands would pass"
    assert error <= bound, f"{what}: {error:.3e}, {bound:.3e} allowed"


def attend(c, q, new, Hkv, scale=0.0, max_len=None, splits=0):
    out = qlin.causal_attention_kv4(q.cuda(), c.dev, i32(starts(new)), max_new=max(new), max_len=max_len, scale=scale, splits=splits, **c.kwargs())
    torch.cuda.synchronize()
    unpacked = plan_text(new, c.length, q.shape[1], Hkv, splits, max(new), max_len).startswith("unpack")
    return out.cpu().double(), unpacked


def set_grid(c, part, grid):
    """Steps and offsets [heads or 1, tokens, 2] of a cache of rooms."""
    grid = grid.to(torch.bfloat16)
    for t in (c.host[part], c.dev[part]):
        t[:, :, :grid.shape[1]] = grid[None].to(t.device)


def check(new, length, Hq=8, Hkv=2, layout="heads", splits=0, seed=0, cache=None, q=None, scale=0.0, max_len=None, by_token=False):
    c = cache or Cache(layout, length, Hkv, seed + 10, spread=0.3)
    q = rand(seed, (sum(new), Hq, HEAD)) if q is None else q
    have, unpacked = attend(c, q, new, Hkv, scale, max_len, splits)
    parts = [[], [], [], []]
    for b, n in enumerate(new):
        m = starts(new)[b]
        for to, x in zip(parts, (have[m:m + n], *errors(f64(q[m:m + n]), c, b, Hkv, scale or HEAD ** -0.5, unpacked))):
            to.append(x)
    parts = [torch.cat(x) for x in parts]
    if by_token:
        for m in range(sum(new)):
            within(*(x[m] for x in parts), f"token {m}")
    else:
        within(*parts, "call")


FORMS = [([1, 1, 1], [300, 77, 600], {}), ([16, 5], [300, 200], {}), ([130], [333], {}), ([100], [333], UNPACKED), ([60, 45], [333, 60], UNPACKED)]


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["heads", "tokens", "packed"])
@pytest.mark.parametrize("splits", [0, 3])
@pytest.mark.parametrize("new,length,kw", FORMS)
def test_error_of_each_form(new, length, kw, splits, layout):
    check(new, length, layout=layout, splits=splits, seed=sum(length), **kw)


def grid_of(size):
    return torch.stack([size, -7.5 * size], -1)[None]


@pytest.mark.gpu
@pytest.mark.parametrize("new,length,kw", FORMS)
def test_error_with_values_of_many_sizes(new, length, kw):
    """Steps of the values with a spread of e^3."""
    Hkv = kw.get("Hkv", 2)
    c = Cache("heads", length, Hkv, 3, spread=0.3)
    set_grid(c, 3, grid_of(0.3 * torch.exp(3 * torch.randn(max(length), generator=torch.Generator().manual_seed(4)))))
    check(new, length, cache=c, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("new,kw", [(16, dict(Hq=32, Hkv=1)), (70, dict(Hq=32, Hkv=1)), (70, UNPACKED)])
def test_error_of_tokens_that_see_ever_larger_rows(new, kw):
    """Keys from 2^-16 and values from 2^-20 on, growing from token to token, so that each new token
    has outputs of its own size."""
    c = Cache("heads", [new], 1, 2, spread=0.3)
    grow = torch.linspace(0, 1, new)
    set_grid(c, 1, grid_of(0.3 * 2.0 ** (16 * grow - 16)))
    set_grid(c, 3, grid_of(0.3 * 2.0 ** (24 * grow - 20)))
    check([new], [new], cache=c, by_token=True, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("new,length,Hq,max_len", [([1, 1], [200, 90], 24, None), ([16, 16], [200, 90], 24, None), ([90, 80], [200, 90], 24, None),
                                                   ([90, 80], [200, 90], 192, 400000)])
def test_error_of_heads_of_different_sizes(new, length, Hq, max_len):
    """Each head of each sequence has keys and values of a size of its own, and queries that bring its scores
    into range."""
    Hkv, G = 3, Hq // 3
    c = Cache("heads", length, Hkv, 7, spread=0.3)
    q = rand(1, (sum(new), Hq, HEAD)).double()
    sizes = [[-14, 3, 9], [12, -8, 0]]
    for b in (0, 1):
        for g in range(Hkv):
            k, v = sizes[b][g], -sizes[b][(g + 1) % 3]
            for t in (c.host, c.dev):
                t[1][b, g] *= 2.0 ** k
                t[3][b, g] *= 2.0 ** v
            q[starts(new)[b]:starts(new)[b + 1], g * G:(g + 1) * G] *= 2.0 ** -k
    q = q.to(torch.bfloat16)
    have, unpacked = attend(c, q, new, Hkv, max_len=max_len)
    assert unpacked == (max_len is not None)
    for b, n in enumerate(new):
        m = starts(new)[b]
        parts = have[m:m + n], *errors(f64(q[m:m + n]), c, b, Hkv, HEAD ** -0.5, unpacked)
        for g in range(Hkv):
            within(*(x[:, g * G:(g + 1) * G] for x in parts), f"sequence {b} head {g}")


# Workgroups of one and of two halves of the keys, alone and in ranges.
SPLIT = [([130], [600], 32, 4, 8, "<1>"), ([60, 70], [300, 600], 64, 2, 12, "<1>"), ([130], [600], 128, 2, 1, "<1>"),
         ([130], [600], 64, 2, 1, "<2>"), ([130], [600], 64, 2, 3, "<2>")]


@pytest.mark.parametrize("new,length,Hq,Hkv,splits,kind", SPLIT)
def test_which_workgroups_a_call_takes(new, length, Hq, Hkv, splits, kind):
    """No launch: forced ranges are planned without a device."""
    text = plan_text(new, length, Hq, Hkv, splits, max_len=100000 if kind == "<2>" else None)
    assert text.startswith("unpack") and f"k_causal_prompt{kind}" in text


@pytest.mark.gpu
@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("new,length,Hq,Hkv,splits,kind", SPLIT)
def test_error_of_workgroups_of_one_and_two_halves(new, length, Hq, Hkv, splits, kind, far):
    """far: rows of keys and values up to 2^16 apart, each with a power of two of its own."""
    c = Cache("heads", length, Hkv, 9, spread=0.3)
    if far:
        g = torch.Generator().manual_seed(2)
        for part in (1, 3):
            set_grid(c, part, grid_of(0.3 * 2.0 ** (-16 * torch.rand(max(length), generator=g))))
    check(new, length, Hq=Hq, Hkv=Hkv, cache=c, splits=splits, seed=1, max_len=100000 if kind == "<2>" else None)

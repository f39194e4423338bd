"""GPU tests of the causal attention where scores are large: keys and queries of powers of two,
whose scores are exact, so that the largest ones share all the weight and the output is their
values' mean (one rounding to bf16, and one of 1 / n: 2 x 2^-8 of the values' size)."""

import numpy as np
import pytest
import torch

from oracle import target_ref as ref
from paper_2607_04244_amd import qlin
from test_target import Cache, f64, i32, rand, starts

pytestmark = pytest.mark.gpu
HEAD = 128

# (new, length, splits, max_len) for each kernel: few, mid<1>, mid<2>, prompt in one half and two
FORMS = [([1, 1], [700, 33], 0, None), ([1, 1], [700, 90], 3, None), ([7], [500], 1, None), ([16, 3], [300, 3], 2, None),
         ([150], [150], 1, None), ([70, 40], [400, 41], 2, None), ([130, 17], [611, 17], 1, 1 << 20), ([90], [300], 2, 1 << 20)]


def case(new, length, Hq, Hkv, seed, size, sign, factor):
    """Scores sign * factor * 2^(2 size) * c_j, c_j in 1 .. 4, of every head; exact in fp32."""
    c = Cache("heads", length, Hkv, seed)
    g = torch.Generator().manual_seed(seed)
    counts = torch.randint(1, 5, c.host[0].shape[:3], generator=g).float()
    c.host[0].zero_()
    c.host[0][..., 3] = (counts * 2.0 ** size).to(torch.bfloat16)
    c.dev[0].copy_(c.host[0])
    q = torch.zeros((sum(new), Hq, HEAD), dtype=torch.bfloat16)
    q[..., 3] = sign * factor * 2.0 ** size
    return c, counts, q


@pytest.mark.parametrize("size", [6, 12, 14, 16, 18, 20, 25, 30, 45, 60])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("factor", [1.0, 1.59375])
def test_the_largest_scores_have_all_the_weight(form, sign, size, factor):
    new, length, splits, max_len = FORMS[form]
    Hq, Hkv = 8, 2
    c, counts, q = case(new, length, Hq, Hkv, 3 + form, size, sign, factor)
    for scale in (0.0, 0.1):
        out = qlin.causal_attention(q.cuda(), *c.dev, i32(starts(new)), max_new=max(new), max_len=max_len, splits=splits, scale=scale, **c.kwargs())
        torch.cuda.synchronize()
        got = f64(out)
        for m, (b, p) in enumerate(ref.positions(new, length)):
            if p < 0:
                continue
            for g in range(Hkv):
                n = sign * counts[b, g, :p + 1].numpy()
                best = n == n.max()
                v = f64(c.host[1][b, g, :p + 1])[best]
                tol = 2 * 2.0 ** -8 * np.abs(v).mean(0) + length[b] * 2.0 ** -24 * np.abs(v).mean(0) + 1e-30
                assert np.all(np.abs(got[m, g * 4:g * 4 + 4] - v.mean(0)) <= tol), (b, p, g)


@pytest.mark.parametrize("form", range(2, len(FORMS)))
def test_rows_beside_one_of_large_scores_keep_their_bits(form):
    """The last new token's queries of every sequence are ordinary, then 2^50 times that."""
    new, length, splits, max_len = FORMS[form]
    c = Cache("heads", length, 2, 4)
    q = rand(form, (sum(new), 8, HEAD), 2.0)
    attend = lambda: qlin.causal_attention(q.cuda(), *c.dev, i32(starts(new)), max_new=max(new), max_len=max_len, splits=splits, **c.kwargs())
    first = attend()
    ends = torch.tensor(starts(new)[1:]) - 1
    q[ends] *= 2.0 ** 50
    second = attend()
    torch.cuda.synchronize()
    keep = torch.ones(sum(new), dtype=torch.bool)
    keep[ends] = False
    assert torch.equal(first[keep.cuda()].view(torch.int16), second[keep.cuda()].view(torch.int16))
    assert torch.isfinite(second).all()


@pytest.mark.parametrize("form", range(len(FORMS)))
def test_scores_of_minus_infinity_alone_give_nan(form):
    """A row whose visible scores are all -infinity has no softmax (0 / 0): NaN; one finite score
    among them has all the weight; a row without visible keys gives zeros."""
    new, length, splits, max_len = FORMS[form]
    c = Cache("heads", length, 2, 5)
    c.host[0].zero_()
    c.host[0][..., 7] = float("-inf")
    c.host[0][:, 1, 1, 7] = 0.0                        # head 1: token 1 has score 0
    c.dev[0].copy_(c.host[0])
    q = torch.zeros((sum(new), 8, HEAD), dtype=torch.bfloat16)
    q[..., 7] = 1.0
    out = qlin.causal_attention(q.cuda(), *c.dev, i32(starts(new)), max_new=max(new), max_len=max_len, splits=splits, **c.kwargs())
    torch.cuda.synchronize()
    got = f64(out)
    for m, (b, p) in enumerate(ref.positions(new, length)):
        assert np.all(np.isnan(got[m, :4])) if p >= 0 else np.all(got[m] == 0)
        if p >= 1:
            assert np.array_equal(got[m, 4:], np.broadcast_to(f64(c.host[1][b, 1, 1]), (4, HEAD)))
        elif p == 0:
            assert np.all(np.isnan(got[m, 4:]))

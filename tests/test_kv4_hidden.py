"""Finite rows behind a token's position in the causal attention over the 4-bit cache (GPU).  The
kernels that read codes keep every bit of earlier tokens' results.  The forms that unpack
bring a head's rows, or each of its rows, into f16's range by powers of two that go by all of a
sequence's rows: there earlier tokens' results stay as exact as they are without the later
rows, within the bound of tests/test_kv4_accuracy.py, though not in every bit."""

import pytest
import torch

from paper_2607_04244_amd import qlin

from test_kv4 import HEAD, Cache, bits, f64, i32, plan_text, rand, starts
from test_kv4_accuracy import errors, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,length,Hq,Hkv,max_len", [([16, 4], [40, 200], 8, 2, None), ([60], [60], 8, 2, None), ([300, 20], [300, 120], 8, 2, None),
                                                       ([70, 20], [70, 120], 64, 1, 100000), ([90], [400], 128, 2, 400000)])
@pytest.mark.parametrize("size", [1e3, -1e5, 1e10, 1e-10, 1e-3, 0.0])
def test_finite_rows_behind_a_token(new, length, Hq, Hkv, max_len, size):
    """Later tokens' rows far larger and far smaller than the ones that are seen, where a head
    changes to powers of two for each row among them."""
    q = rand(1, (sum(new), Hq, HEAD))
    c = Cache("heads", length, Hkv, 4, spread=0.3)
    unpacked = plan_text(new, length, Hq, Hkv, 0, max(new), max_len).startswith("unpack")
    assert unpacked == (max_len is not None)
    outs = []
    for junk in (False, True):
        dev = [t.clone() for t in c.dev]
        if junk:
            for b, (n, L) in enumerate(zip(new, length)):
                cut = L - n + n // 2 + 1              # hidden from the first half of the new tokens
                for part in (1, 3):
                    dev[part][b, :, cut:, 0] = size
                    dev[part][b, :, cut:, 1] = -3 * size
        outs.append(qlin.causal_attention_kv4(q.cuda(), dev, i32(starts(new)), i32(length), max_new=max(new), max_len=max_len))
    torch.cuda.synchronize()
    m = 0
    for b, n in enumerate(new):
        first = [out[m:m + n // 2 + 1] for out in outs]
        if unpacked:
            parts = [x[:n // 2 + 1] for x in errors(f64(q[m:m + n]), c, b, Hkv, HEAD ** -0.5, True)]
            for out in first:
                within(out.cpu().double(), *parts, f"sequence {b}")
        else:
            assert torch.equal(bits(first[0]), bits(first[1]))
        m += n

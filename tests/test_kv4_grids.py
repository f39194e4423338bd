"""The causal attention over 4-bit rows whose grids a caller made: steps of either sign, tiny steps
beside constant rows (GPU).  A row is step c + offset for any bf16 step and offset; errors are held
to what roundings add up to, as derived in tests/test_kv4_accuracy.py."""

import pytest
import torch

from test_kv4 import HEAD, UNPACKED, Cache, f64, rand
from test_kv4_accuracy import attend, check, errors, set_grid

pytestmark = pytest.mark.gpu

FORMS = [(1, dict(Hq=8, Hkv=1)), (16, dict(Hq=8, Hkv=1)), (300, dict(Hq=8, Hkv=1)), (60, UNPACKED)]


@pytest.mark.parametrize("power", [-60, -30, -14, 0, 10, 20, 40])
@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("new,kw", FORMS)
def test_steps_of_either_sign(new, kw, mixed, power):
    """Values whose steps are negative, all or in turn, from sizes that vanish in f16 to ones past it; the
    keys' as well, of ordinary size."""
    L = 333
    c = Cache("heads", [L], 1, power + 100, spread=0.3)
    g = torch.Generator().manual_seed(power + 200)
    sign = torch.where(torch.rand(L, generator=g) < 0.5, -1.0, 1.0) if mixed else -torch.ones(L)
    for part, size in ((1, 0.3), (3, 2.0 ** power)):
        step = sign * size * torch.exp(0.3 * torch.randn(L, generator=g))
        set_grid(c, part, torch.stack([step, -7 * step + 0.3 * size * torch.randn(L, generator=g)], -1)[None])
    check([new], [L], cache=c, seed=power + 300, **kw)


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("step,offset", [(-100, 28), (-110, 50), (-90, 55), (-120, 1)])
@pytest.mark.parametrize("new,kw", FORMS)
def test_tiny_steps_beside_constant_rows(new, kw, step, offset, order):
    """Every fifth row is constant (step 0) and large, the others' steps are tiny: weights held for
    those must not take the offsets past fp32.  All values count with one sign, so errors are relative
    to the result: its rounding 2^-8, weights 2^-12, sums of 333 2^-15; scores move by 140 x 2^-24 scale sum|q|
    (15 s + |o|) < 140 x 2^-24 x 0.0884 x 150 x 8 < 2^-10 and, where keys are rounded to f16, by 2^-12 scale sum|q||k| <
    2^-12 x 0.0884 x 150 x 4 < 2^-6: twice that, so less than 2^-4."""
    L = 333
    c = Cache("heads", [L], 1, 5, spread=0.3)
    grid = torch.zeros(L, 2)
    grid[:, 0] = 2.0 ** step
    grid[:, 1] = -7 * 2.0 ** step
    g = torch.Generator().manual_seed(1)
    where = torch.arange(0, L, 5) if order > 0 else L - 1 - torch.arange(0, L, 5)
    grid[where, 0] = 0.0
    grid[where, 1] = 2.0 ** offset * torch.randn(len(where), generator=g).abs()
    # a constant row has one value for all dimensions; with it at both ends every token sees one
    grid[0], grid[-1] = torch.tensor([0.0, 2.0 ** offset]), torch.tensor([0.0, 2.0 ** offset])
    set_grid(c, 3, grid[None])
    q = rand(6, (new, kw["Hq"], HEAD))
    have, unpacked = attend(c, q, [new], 1, max_len=kw.get("max_len"))
    want = errors(f64(q), c, 0, 1, HEAD ** -0.5, unpacked)[0]
    assert want.min() > 0 and ((have - want).abs() <= 2.0 ** -4 * want).all()

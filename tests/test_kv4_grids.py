"""The causal attention over 4-bit rows whose grids a caller made: steps of either sign
(GPU).  A row is step c + offset for any bf16 step and offset; errors are held
to what roundings add up to, as derived in tests/test_kv4_accuracy.py."""

import pytest
import torch

from test_kv4 import UNPACKED, Cache
from test_kv4_accuracy import check, set_grid

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

"""Seeded random batches through the target's operators, every output element against the
64-bit oracle (the bounds are those of tests/test_target.py): sizes, head groups, layouts,
key ranges, declared bounds and padding in combinations that no list names."""

import random

import pytest

from test_target import LAYOUTS, check_append, check_attention, check_verify, verify_case

pytestmark = pytest.mark.gpu


def batch(rng, most_new, most_old, sequences):
    new = [0 if rng.random() < 0.1 else int(2 ** rng.uniform(0, most_new)) for _ in range(sequences)]
    length = [max(n + rng.choice([0, 0, int(2 ** rng.uniform(0, most_old))]) - (rng.random() < 0.05) * 3, 0) for n in new]
    if not any(new):
        new[0], length[0] = 1, max(length[0], 1)
    return new, length


@pytest.mark.parametrize("seed", range(48))
def test_attention_sweep(seed):
    rng = random.Random(1000 + seed)
    few = seed % 3                          # single tokens, blocks, prompts
    new, length = batch(rng, (0.9, 4.2, 8.5)[few], (10.5, 10, 9.5)[few], rng.choice([1, 2, 3, 7]))
    Hkv = rng.choice([1, 2, 3, 8])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 5, 8])
    if few == 2 and Hq * sum(new) > 4000:
        Hq, Hkv = 4, 1
    check_attention(new, length, rng.choice(LAYOUTS), Hq=Hq, Hkv=Hkv, splits=rng.choice([0, 0, 1, 2, 3, 6]), seed=seed, pad=rng.choice([0, 0, 5]),
                    fused=rng.random() < 0.3, max_len=rng.choice([None, None, max(length), 1 << 20]),
                    max_new=rng.choice([None, None, None, sum(new)]), sigma=rng.choice([0.5, 2.0, 6.0]))


@pytest.mark.parametrize("seed", range(24))
def test_append_sweep(seed):
    rng = random.Random(2000 + seed)
    new, length = batch(rng, rng.choice([1, 5, 9]), 9, rng.choice([1, 2, 5, 70]))
    Hkv = rng.choice([1, 2, 4])
    fused = rng.random() < 0.5
    check_append(new, length, rng.choice(LAYOUTS) if len(new) <= 7 else "packed", Hq=Hkv * rng.choice([1, 2, 3, 4]), Hkv=Hkv,
                 norm=rng.random() < 0.7, rot=rng.choice([0, 16, 48, 64, 128, 128]), interleaved=rng.random() < 0.4, pad=rng.choice([0, 3]),
                 fused=fused, in_place=rng.random() < 0.4, theta=rng.choice([1e4, 1e6]), seed=seed)


@pytest.mark.parametrize("seed", range(24))
def test_verify_sweep(seed):
    rng = random.Random(3000 + seed)
    n, drafts, V = rng.choice([1, 2, 5, 33]), rng.choice([0, 1, 3, 7, 15, 20]), int(2 ** rng.uniform(0, 13.5))
    target, draft, drafted, u = verify_case(n, drafts, V, seed, near=rng.choice([0.05, 0.4, 2.0]), with_draft=rng.random() < 0.6)
    kw = {}
    if rng.random() < 0.5:
        kw["T"] = [rng.choice([0.0, 0.5, 1.0, 1.7]) for _ in range(n)]
    if rng.random() < 0.5:
        kw["count"] = [rng.randint(0, drafts) for _ in range(n)]
    check_verify(target, draft, drafted, u, **kw)

"""What a call of the target's operators writes must not lie on any array it reads, the small
ones included (CPU: refused before any HIP call)."""

import pytest

from paper_2607_04244_amd import qlin
from test_target_abi import A, INVALID, STEP, append, attend, batch, cache

OUT, K, V, WS = A + 6 * STEP, A + STEP, A + 2 * STEP, A + 7 * STEP      # the calls' defaults
ARRAYS = ("new_start", "length", "cache_start")


@pytest.mark.parametrize("at", [OUT, OUT + 4096, K + 512, V, V + 1024])
@pytest.mark.parametrize("name", ARRAYS)
def test_append_refuses_lengths_on_what_it_writes(name, at):
    assert append(b=batch(**{name: at})) == INVALID and "overlap" in qlin.last_error()


@pytest.mark.parametrize("at", [OUT, OUT + 4096, K, V + 256])
@pytest.mark.parametrize("name", ["qn", "kn", "freq"])
def test_append_refuses_weights_on_what_it_writes(name, at):
    assert append(**{name: at}) == INVALID and "overlap" in qlin.last_error()


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("at", [OUT, OUT + 4096])
@pytest.mark.parametrize("name", ARRAYS)
def test_attention_refuses_lengths_on_its_output(name, at, splits):
    assert attend(b=batch(**{name: at}), splits=splits) == INVALID and "overlap" in qlin.last_error()


@pytest.mark.parametrize("name", ARRAYS)
def test_attention_refuses_lengths_on_its_workspace(name):
    assert attend(b=batch(**{name: WS + 64}), splits=3) == INVALID and "overlap" in qlin.last_error()


def test_ends_that_touch_are_no_overlap():
    """Behind the last byte written: refused for the missing workspace, which is checked later."""
    rows, wide = 40, 4096
    end = OUT + rows * wide * 2
    for name in ARRAYS:
        assert attend(b=batch(**{name: end}), splits=3, ws=None, wb=0) == INVALID and "workspace" in qlin.last_error()

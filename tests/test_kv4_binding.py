"""The Python binding's reading of 4-bit caches (CPU: what it makes of shapes and strides, no
call)."""

import pytest
import torch

from paper_2607_04244_amd import qlin


@pytest.fixture(autouse=True)
def cpu(monkeypatch):
    monkeypatch.setattr(qlin, "_torch", torch)


def new(*shape):
    return qlin.new_kv4_cache(*shape, device="cpu")


def read(cache):
    """(heads, slots, token stride, head stride, slots between sequences, capacity); -1: the CPU's device index."""
    c = qlin._kv4_cache(cache, -1)
    return c.heads, c.slots, c.token_stride, c.head_stride, c.seq_slots, c.capacity


def test_layouts():
    assert read(new(3, 2, 40)) == (2, 2 * 80 + 40, 1, 40, 80, 40)
    assert read(new(50, 4)) == (4, 50, 4, 1, 0, 0)
    assert read([t.transpose(1, 2) for t in new(3, 40, 2)]) == (2, 120, 2, 1, 40, 40)
    assert read([t[:, :2] for t in new(50, 4)]) == (2, 50, 4, 1, 0, 0)
    assert read([t[:, 1:, 5:30] for t in new(3, 4, 40)]) == (3, 2 * 160 + 25, 1, 40, 160, 25)


def test_dimensions_of_one_may_have_any_stride():
    assert read([t.expand(1, 2, 40, t.shape[-1]) for t in new(1, 2, 40)])[:2] == (2, 40)
    assert read([t[:, :1] for t in new(50, 4)]) == (1, 50, 4, 1, 0, 0)
    assert read([t[:, :, :1] for t in new(3, 2, 40)])[5] == 1


@pytest.mark.parametrize("shape,own", [((3, 4, 40), (3, 1, 40)), ((3, 4, 40), (3, 4, 1)), ((3, 4, 40), (1, 1, 1)),
                                       ((50, 4), (50, 1)), ((50, 4), (1, 4))])
def test_expanded_caches_are_refused(shape, own):
    """Heads or tokens that share memory by a stride of 0 have no rows of their own: taken as a row
    apart they would lie behind the cache."""
    with pytest.raises(ValueError, match="whole"):
        read([t.expand(*shape, t.shape[-1]) for t in new(*own)])


def test_sequences_may_share_a_room():
    """As with a bf16 cache: one room for all."""
    assert read([t.expand(3, 4, 40, t.shape[-1]) for t in new(1, 4, 40)]) == (4, 40, 1, 40, 0, 40)

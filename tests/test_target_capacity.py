"""A sequence's room in the target's cache: lengths past the capacity count as no cached
tokens, in every layout, and touch no other head's or sequence's slots."""

import numpy as np
import pytest
import torch

from paper_2607_04244_amd import qlin
from test_target_abi import INVALID, UNSUPPORTED, append, attend, cache

HEAD = 128


@pytest.mark.parametrize("call", [append, attend])
def test_capacity_is_checked(call):
    fields = [getattr(cache(), n) for n, _ in qlin.KVCache._fields_]
    assert qlin.KVCache(*fields).capacity == 0 and qlin.KVCache(*fields).k == cache().k
    room = lambda n: qlin.KVCache(*fields, capacity=n)
    assert room(512).capacity == 512 and room(512).seq_slots == cache().seq_slots
    assert call(c=room(-1)) == INVALID and call(c=room((1 << 40) + 1)) == UNSUPPORTED
    assert call(c=room(512), D=64) == UNSUPPORTED                    # checked behind the cache: its capacity passed


def test_binding_gives_the_capacity_of_a_cache_of_sequences(monkeypatch):
    monkeypatch.setattr(qlin, "_torch", torch)
    on_host = -1
    t = torch.zeros((3, 2, 40, HEAD), dtype=torch.bfloat16)
    wide = torch.zeros((3, 2, 64, HEAD), dtype=torch.bfloat16)[:, :, :40]
    for c in (t, t.transpose(1, 2).contiguous().transpose(1, 2), wide, t.transpose(0, 1).contiguous().transpose(0, 1), t[:1], t[:1].expand(3, 2, 40, HEAD)):
        assert qlin._kv_cache(c, c, on_host).capacity == 40
    assert qlin._kv_cache(t[0].transpose(0, 1), t[0].transpose(0, 1), on_host).capacity == 0


def layouts(n, heads, cap, seed):
    """(name, storage, [n, heads, cap, 128] view) of caches that lie differently; slots outside the
    view hold values too."""
    g = torch.Generator().manual_seed(seed)
    make = lambda *shape: torch.randn(shape, generator=g).to(torch.bfloat16).cuda()
    s = make(n, heads, cap, HEAD)
    yield "heads", s, s
    s = make(n, cap, heads, HEAD)
    yield "tokens", s, s.transpose(1, 2)
    s = make(heads, n, cap, HEAD)
    yield "heads first", s, s.transpose(0, 1)
    s = make(n, heads, cap + 9, HEAD)
    yield "a part of the capacity", s, s[:, :, :cap]
    s = make(2 * n, cap, heads, HEAD)
    yield "every second sequence", s, s[::2].transpose(1, 2)


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(5))
@pytest.mark.parametrize("starts", [None, "same", "inside"])
@pytest.mark.parametrize("over", [1, 7, 1 << 20])
@pytest.mark.parametrize("new", [[1, 1, 1], [3, 2, 4], [40, 5, 33]])
def test_lengths_past_the_capacity(which, starts, over, new):
    """Sequence 0 is too long, 1 fills its room exactly, 2 has less; with cache_start, sequences
    at the starts of their rooms (in another order), or 5 slots into them."""
    n, heads, cap, Hq = 3, 2, 70, 4
    (_, ks, kc), (_, vs, vc) = (list(layouts(n, heads, cap, seed))[which] for seed in (1, 2))
    into = 5 if starts == "inside" else 0
    length = [cap - into + over, cap - into, cap - into - 9]
    room = [0, 1, 2] if starts is None else [1, 2, 0]
    seq_slots = kc.stride(0) // kc.stride(2)
    at = None if starts is None else torch.tensor([r * seq_slots + into for r in room], dtype=torch.int64, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    batch = dict(new_start=i32([0, *np.cumsum(new).tolist()]), length=i32(length), max_new=max(new), cache_start=at)
    M = sum(new)
    g = torch.Generator().manual_seed(3)
    rows = [torch.randn((M, h * HEAD), generator=g).to(torch.bfloat16).cuda() for h in (Hq, heads, heads)]
    want_k, want_v = ks.clone(), vs.clone()
    view = lambda want: torch.as_strided(want, kc.shape, kc.stride())
    m = new[0]
    for b in (1, 2):                                                   # no norm, no rotation: copies
        for i in range(new[b]):
            slot = into + length[b] - new[b] + i
            view(want_k)[room[b], :, slot] = rows[1][m].view(heads, HEAD)
            view(want_v)[room[b], :, slot] = rows[2][m].view(heads, HEAD)
            m += 1
    q = qlin.norm_rope_append(*rows, kc, vc, **batch)
    out = qlin.causal_attention(q, kc, vc, **batch)
    torch.cuda.synchronize()
    assert torch.equal(ks, want_k) and torch.equal(vs, want_v)
    assert torch.equal(q.view(M, -1), rows[0])
    assert torch.all(out[:new[0]] == 0) and torch.all(out[new[0]:].abs().sum((1, 2)) > 0)
    # the two others as without the first
    alone = qlin.causal_attention(q[new[0]:].contiguous(), kc, vc, **{**batch, "new_start": batch["new_start"][1:] - new[0],
                                                                      "length": batch["length"][1:].contiguous(),
                                                                      "cache_start": torch.tensor([r * seq_slots + into for r in room[1:]], device="cuda")})
    torch.cuda.synchronize()
    assert torch.all((out[new[0]:].float() - alone.float()).abs() <= 2.0 ** -6 * alone.float().abs() + 2.0 ** -7)

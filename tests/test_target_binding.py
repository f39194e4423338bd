"""The Python binding's reading of tensors for the target's operators (CPU: what it makes of
shapes and strides, no call)."""

import sys

import pytest
import torch

from paper_2607_04244_amd import qlin

BF16 = torch.bfloat16


@pytest.mark.parametrize("n,rows", [(1, 1), (1, 4), (3, 1), (3, 4)])
def test_logits_need_contiguous_rows_whatever_their_number(n, rows):
    """A single row too: a column of vocabulary-major logits, every second logit, one logit
    expanded."""
    V = 50
    base = torch.zeros((n, rows, 2 * V), dtype=BF16)
    assert qlin._logit_rows("t", base[:, :, :V], n, rows, V) == (2 * V if n * rows > 1 else V)
    assert qlin._logit_rows("t", base[:, :, :1], n, rows, 1) >= 1
    assert qlin._logit_rows("t", base[:, :0, :V], n, 0, V) == V                    # no rows
    major = torch.zeros((V, n, rows, 2), dtype=BF16)[..., 1].permute(1, 2, 0)
    for t in (base[:, :, ::2], torch.zeros((n, rows, 1), dtype=BF16).expand(n, rows, V), major):
        with pytest.raises(ValueError, match="contiguous rows"):
            qlin._logit_rows("t", t, n, rows, V)


def test_a_second_thread_in_the_first_call_finds_what_it_needs(monkeypatch):
    """At every instruction of the first call's look at torch, another call finds the current
    stream's getter set, or sets it."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    for name in ("_torch", "_current_device", "_raw_stream"):
        monkeypatch.setattr(qlin, name, None)
    state, seen = ("_torch", "_current_device", "_raw_stream"), []

    def at_each_instruction(frame, event, arg):
        frame.f_trace_opcodes = True
        if event == "opcode":
            sys.settrace(None)
            before = [getattr(qlin, n) for n in state]
            assert qlin._device() == 0
            seen.append(all(getattr(qlin, n) is not None for n in state))
            for n, v in zip(state, before):
                setattr(qlin, n, v)
            sys.settrace(trace)
        return at_each_instruction

    def trace(frame, event, arg):
        return at_each_instruction(frame, event, arg) if frame.f_code is qlin._device.__code__ else None

    sys.settrace(trace)
    try:
        qlin._device()
    finally:
        sys.settrace(None)
    assert len(seen) > 10 and all(seen)

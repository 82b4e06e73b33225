"""What aal_beam_reorder checks before it launches anything, on the CPU: its tensors
claim to be on a device, and the library's entry point is a stand-in that keeps its arguments."""
import contextlib
import struct

import pytest
import torch

from paper_2609_24150_amd import api


class OnDevice(torch.Tensor):
    is_cuda = True


def on(t):
    return t.as_subclass(OnDevice)


@pytest.fixture
def calls(monkeypatch):
    made = []

    class Lib:
        @staticmethod
        def aal_beam_reorder(table, n_states, B, W, n, parents, stream):
            rows = struct.unpack(f"{n_states * 10}q", table)
            made.append([rows[i:i + 10] for i in range(0, len(rows), 10)])
            return 0

    monkeypatch.setattr(api._lib, "lib", lambda: Lib)
    monkeypatch.setattr(api, "_guard", lambda *a: contextlib.nullcontext())
    monkeypatch.setattr(api, "_raw_stream", lambda *a: 0)
    return made


def test_parents_inside_of_what_is_written(calls):
    """Back-pointers [T, B, W] that are a state themselves, the last step's the parents."""
    T, B, W = 5, 2, 4
    back = on(torch.zeros(T, B, W, dtype=torch.int32))
    state, other = back.permute(1, 2, 0), on(torch.zeros(T, B, W, dtype=torch.int32)).permute(1, 2, 0)
    for t in range(T):
        for states, out in (([state], None), ([other, state], None), ([other], [state]), ([other, other], [other.clone(), state])):
            with pytest.raises(ValueError, match="parents"):
                api.aal_beam_reorder(states, back[t], out=out)
    assert not calls
    # what is only read may hold them, and so may the steps that are not moved
    api.aal_beam_reorder([state], back[1], out=[other])
    api.aal_beam_reorder([back[:2].permute(1, 2, 0), other], back[2])
    api.aal_beam_reorder([back[3:].permute(1, 2, 0), back[:2].permute(1, 2, 0)], back[2])
    # a state without bytes writes nothing
    api.aal_beam_reorder([state[:, :, :0]], back[0])
    assert len(calls) == 4


def test_parents_of_the_call_before_in_one_buffer(calls):
    """Parents and a state in one buffer, end to end."""
    B, W, L = 2, 4, 6
    pool = on(torch.zeros(B * W * (L + 1) + 1, dtype=torch.int32))
    state = pool[:B * W * L].view(B, W, L)
    api.aal_beam_reorder([state], pool[B * W * L:-1].view(B, W))
    with pytest.raises(ValueError, match="parents"):
        api.aal_beam_reorder([state], pool[B * W * L - 1:-2].view(B, W))
    assert len(calls) == 1

"""CPU check of aal_beam_reorder: states of more bytes than any memory holds are refused, where the
number of workgroups would pass 64 bits and launches would not end."""
import os

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2609_24150_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.fail("libaal.so is not built (run __graft_entry__.build())")
    return _lib


@pytest.mark.parametrize("B,W,segments,size", [(1 << 29, 2, 1 << 38, 1), (1 << 24, 8, 1, 1 << 38), (1 << 29, 2, 1, (1 << 20) + 1)])
def test_more_than_any_memory(L, B, W, segments, size):
    table = (L.BeamState * 1)(L.BeamState(16, None, 0, 0, 0, 0, 0, 0, segments, size))
    assert L.lib().aal_beam_reorder(table, 1, B, W, W, 16, None) == 1
    assert "2^50" in L.lib().aal_last_error().decode()

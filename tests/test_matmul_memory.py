"""aal_fp8_matmul refuses outputs and workspaces in its operands' memory, before anything is launched: on the CPU, with
tensors that claim to be on a device and a stand-in for the library."""
import contextlib

import pytest
import torch

from paper_2609_24150_amd import api


class OnDevice(torch.Tensor):
    is_cuda = True


@pytest.fixture
def calls(monkeypatch):
    made = []

    class Lib:
        aal_fp8_matmul = staticmethod(lambda *a: made.append(a) or 0)
        aal_fp8_matmul_workspace_bytes = staticmethod(lambda *a: 256)

    monkeypatch.setattr(api._lib, "lib", lambda: Lib)
    monkeypatch.setattr(api, "_guard", lambda *a: contextlib.nullcontext())
    monkeypatch.setattr(api, "_raw_stream", lambda *a: 0)
    api.aal_fp8_matmul_workspace_bytes.cache_clear()
    yield made
    api.aal_fp8_matmul_workspace_bytes.cache_clear()


def test_outputs_and_workspaces_apart(calls):
    pool = torch.zeros(1 << 14, dtype=torch.uint8)
    shift = -pool.data_ptr() % 16
    piece = lambda at, n, dtype: pool[shift + at:shift + at + n].view(dtype).as_subclass(OnDevice)  # noqa: E731
    a = piece(0, 4 * 128, torch.float8_e4m3fn).view(4, 128)
    b = piece(1024, 6 * 128, torch.float8_e4m3fn).view(6, 128)
    sa, sb = piece(2048, 16, torch.float32).view(4, 1), piece(3072, 24, torch.float32).view(6, 1)
    own = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)  # noqa: E731
    for at in (0, 512 - 16, 1024 + 768 - 16, 2048, 3072 + 16, 2048 - 80):
        with pytest.raises(ValueError, match="share no memory"):
            api.aal_fp8_matmul(a, sa, b, sb, out=piece(at, 96, torch.float32).view(4, 6))
        with pytest.raises(ValueError, match="share no memory"):
            api.aal_fp8_matmul(a, sa, b, sb, ws=piece(at, 256, torch.uint8))
    with pytest.raises(ValueError, match="share no memory"):
        api.aal_fp8_matmul(a, sa, b, sb, out=piece(4096, 96, torch.float32).view(4, 6), ws=piece(4096 + 80, 256, torch.uint8))
    assert not calls
    api.aal_fp8_matmul(a, sa, b, sb, out=piece(512, 96, torch.float32).view(4, 6), ws=piece(608, 256, torch.uint8))
    api.aal_fp8_matmul(a, sa, a, sa, out=own(4, 4), ws=own(256, dtype=torch.uint8))
    api.aal_fp8_matmul(a, sa, b, sb)
    assert len(calls) == 3

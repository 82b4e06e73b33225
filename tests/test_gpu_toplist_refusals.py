"""What aal_topk_loss_fwd_bwd refuses of the tensors that it hands on as bare addresses: a workspace
or a scale that the device cannot use ends in an exception, not in the kernel."""
import pytest
import torch

import test_gpu_topk_loss as loss

pytestmark = pytest.mark.gpu

F32 = torch.float32
A = loss.A


def test_workspaces_and_scales(A):
    zd, top, ids, rest = loss.make(2, 3, 100, 5, F32, 1)
    call = lambda **kw: A.aal_topk_loss_fwd_bwd(zd, top, ids, 3, rest=rest, weights=loss.WEIGHTS["all"], **kw)  # noqa: E731
    n = A.aal_topk_loss_workspace_bytes(A.AAL_LAYOUT_WINDOWS, 2, 3, 3)
    want = call()
    good = torch.empty(n, dtype=torch.uint8, device="cuda")
    for ws in (good, torch.empty(n + 512, dtype=torch.uint8, device="cuda")):
        assert torch.equal(call(ws=ws)["grad"], want["grad"])
    for ws in (torch.empty(n, dtype=torch.uint8), good[:1].expand(n), torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            call(ws=ws)
    for scale in (torch.ones(0, device="cuda"), torch.ones(1)):
        with pytest.raises((ValueError, TypeError)):
            call(grad_scale=scale)
    got = call(grad_scale=torch.full((1,), 2.0, device="cuda"))
    assert torch.equal(got["grad"], 2 * want["grad"])

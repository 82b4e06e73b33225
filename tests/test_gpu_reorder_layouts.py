"""aal_beam_reorder between layouts: narrowed caches and contiguous tensors, layers as
views of one tensor, refused parents.  Moved bytes are compared for equality."""
import pytest
import torch

from test_gpu_beam import A, BF16  # noqa: F401

pytestmark = pytest.mark.gpu


def taken(state, parents):
    return state[torch.arange(parents.shape[0], device="cuda")[:, None], parents.long()]


@pytest.mark.parametrize("dtype", [BF16, torch.uint8, torch.int64])
@pytest.mark.parametrize("W,n", [(3, 4), (4, 4), (20, 33), (64, 128)])
def test_narrowed_and_contiguous(A, W, n, dtype):  # noqa: F811
    B, heads, length, dim = 2, 3, 9, 5
    g = torch.Generator("cuda").manual_seed(n)
    make = lambda k, *s: torch.randint(0, 120, (B, k, *s), generator=g, device="cuda").to(dtype)  # noqa: E731
    parents = torch.randint(0, W, (B, n), generator=g, device="cuda", dtype=torch.int32)
    cache, dense = make(W, heads, length, dim), make(W, heads, 4, dim)
    to_dense, to_cache = make(n, heads, 4, dim), make(n, heads, length, dim)
    before = to_cache.clone()
    A.aal_beam_reorder([cache[:, :, :, 2:6], dense], parents, out=[to_dense, to_cache[:, :, :, 1:5]])
    assert torch.equal(to_dense, taken(cache[:, :, :, 2:6], parents))
    assert torch.equal(to_cache[:, :, :, 1:5], taken(dense, parents))
    assert torch.equal(to_cache[:, :, :, :1], before[:, :, :, :1]) and torch.equal(to_cache[:, :, :, 5:], before[:, :, :, 5:])


def test_layers_of_one_tensor(A):  # noqa: F811
    """100 layers of [B, W, layers, heads, length, dim], some positions of each, in place, with parents out of range too."""
    B, W, n = 2, 4, 100
    g = torch.Generator("cuda").manual_seed(3)
    t = torch.randn(B, W, n, 2, 12, 8, generator=g, device="cuda").to(BF16)
    parents = torch.tensor([[1, 0, 3, 3], [-1, 0, 4, 2]], dtype=torch.int32, device="cuda")
    kept = torch.where((parents >= 0) & (parents < W), parents, torch.arange(W, dtype=torch.int32, device="cuda"))
    want = t.clone()
    want[..., 3:9, :] = taken(t, kept)[..., 3:9, :]
    A.aal_beam_reorder([v[:, :, :, 3:9] for v in t.unbind(2)], parents)
    assert torch.equal(t, want)


def test_back_pointers_with_parents_of_their_own(A):  # noqa: F811
    """Back-pointers [steps, B, W] reordered by their last step: a copy of it is taken, its own memory is refused."""
    T, B, W = 6, 2, 4
    g = torch.Generator("cuda").manual_seed(1)
    back = torch.randint(0, W, (T, B, W), generator=g, device="cuda", dtype=torch.int32)
    before = back.clone()
    for t in range(T):
        with pytest.raises(ValueError):
            A.aal_beam_reorder([back.permute(1, 2, 0)], back[t])
    torch.cuda.synchronize()
    assert torch.equal(back, before)
    A.aal_beam_reorder([back.permute(1, 2, 0)], back[-1].clone())
    assert torch.equal(back.permute(1, 2, 0), taken(before.permute(1, 2, 0), before[-1]))

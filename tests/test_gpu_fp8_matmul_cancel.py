"""aal_fp8_matmul where large products cancel between groups of eight neighbours, against
the error that include/aal.h states: fp32 results are sums in fp32; bf16 results are off by
7 2^-13 of sum |sa sb a b| besides, and are rounded to bf16.

fp32: 128 additions of a block of at most 2^-23 of its sum of magnitudes each, the scales and the blocks' sums
2^-24 each.  The values here are whole numbers under 2^24, so the exact results are theirs."""
import pytest
import torch

from test_gpu_fp8_matmul import A, BF16, F32  # noqa: F401

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


def groups(rows, K, small, seed):
    """Eights of one value of +-448 and seven of +-small: the large ones cancel between neighbouring eights, the small ones
    add up."""
    g = torch.Generator().manual_seed(seed)
    x = torch.full((rows, K), float(small))
    at = torch.randint(0, 8, (1, K // 8), generator=g).expand(rows, -1)
    large = torch.full((rows, K // 8), 448.0)
    x.view(rows, K // 8, 8).scatter_(2, at[..., None], large[..., None])
    return x


@pytest.mark.parametrize("M,N,K", [(4, 130, 512), (32, 300, 4096), (150, 300, 1024), (150, 33001, 512), (300, 4000, 16384)])
@pytest.mark.parametrize("small_a,small_b", [(15, 1), (3, 5), (30, 1), (1, 1), (240, 120)])
def test_large_products_that_cancel(A, M, N, K, small_a, small_b):  # noqa: F811
    a = groups(M, K, small_a, 1)
    b = groups(N, K, small_b, 1)  # the large ones at the same places
    b.view(N, K // 16, 2, 8)[:, :, 1] = torch.where(b.view(N, K // 16, 2, 8)[:, :, 1] == 448, -448.0, float(small_b))
    x, y = a.cuda(), b.cuda()
    want = x.double() @ y.double().t()
    mag = x.double().abs() @ y.double().abs().t()
    q, r = (t.to(E4M3).contiguous() for t in (x, y))
    sa, sb = (torch.ones(t.shape[0], K // 128, device="cuda") for t in (x, y))
    blocks = K // 128
    fp32 = (128 * 2.0 ** -23 + (blocks + 2) * 2.0 ** -24) * mag
    assert ((A.aal_fp8_matmul(q, sa, r, sb, out_dtype=F32).double() - want).abs() <= fp32).all()
    tol = fp32 + 7 * 2.0 ** -13 * mag
    off = (A.aal_fp8_matmul(q, sa, r, sb, out_dtype=BF16).double() - want).abs()
    assert (off <= tol + 2.0 ** -8 * (want.abs() + tol)).all(), (off / mag).max().item()

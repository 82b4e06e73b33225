"""aal_fp8_matmul with scales whose product, or whose products with single values, fp32 does
not hold while the results are ordinary numbers, against the fp64 oracle.

Tolerances are those of test_gpu_fp8_matmul.py: a block's sum takes the two scales with one rounding more at
most, which is counted there as that of the scales' product."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as H

from test_gpu_fp8_matmul import A, BF16, E8M0, F32, check, operand  # noqa: F401

pytestmark = pytest.mark.gpu

# few rows; tiles of 128 x 128, in parts too; tiles of 256 x 256 where results are bf16
SIZES = [(5, 300, 700), (20, 200, 1100), (150, 300, 700), (140, 130, 4000), (140, 33001, 700)]


def powers(shape, least, most, scale, seed):
    g = torch.Generator().manual_seed(seed)
    s = torch.exp2(torch.randint(least, most + 1, shape, generator=g).float())
    if scale == F32:
        s = s * (1 + torch.rand(shape, generator=g))
    return s.to(scale).cuda()


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("scale", [F32, E8M0])
@pytest.mark.parametrize("block", [1, 128])
def test_zeros_under_large_scales(A, M, N, K, out, scale, block):  # noqa: F811
    """Blocks of zeros whose scales' product overflows, between ordinary ones."""
    a, b = operand(M, K, "e4m3", scale, 1, 1), operand(N, K, "e5m2", scale, block, 2)
    sa, sb = a[1].float(), b[1].float()
    for j in range(1, sa.shape[1], 2):
        a[0].view(torch.uint8)[:, j * 128:(j + 1) * 128] = 0x80 if j % 4 == 1 else 0
        sa[:, j], sb[:, j] = 2.0 ** 100, 2.0 ** (28 if j % 4 == 1 else 120)
    a, b = (a[0], sa.to(scale)), (b[0], sb.to(scale))
    check(A.aal_fp8_matmul(*a, *b, out_dtype=out), a, b, out)


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("scale", [F32, E8M0])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("fmt,high,low", [("e4m3", 64, -70), ("e5m2", 68, -76)])
def test_products_of_scales_beyond_fp32(A, M, N, K, out, scale, block, fmt, high, low):  # noqa: F811
    """Denormal values (7 2^-9 of e4m3, 3 2^-16 of e5m2 at most) under scales of 2^128 and more together, normal ones under
    2^-136 and less: sums of large and of small, but ordinary numbers."""
    for least, mask in ((high, 0x83 if fmt == "e5m2" else 0x87), (low, 0xff)):
        a, b = operand(M, K, fmt, scale, 1, 3), operand(N, K, fmt, scale, block, 4)
        for v in (a[0], b[0]):
            v.view(torch.uint8).bitwise_and_(mask)
            if mask == 0xff:  # values of 2^6 to 2^7, of 2^11 to 2^13
                u = v.view(torch.uint8)
                u.bitwise_and_(0x87).bitwise_or_(0x68)
        sa, sb = powers(a[1].shape, least, least + 1, scale, 5), powers(b[1].shape, least, least + 1, scale, 6)
        a, b = (a[0], sa), (b[0], sb)
        check(A.aal_fp8_matmul(*a, *b, out_dtype=out), a, b, out)


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("scale", [F32, E8M0])
@pytest.mark.parametrize("block", [1, 128])
def test_single_products_beyond_fp32(A, M, N, K, out, scale, block):  # noqa: F811
    """Ones under scales of 2^-127 together, whose sums are normal numbers, and values of 448 that cancel in
    pairs under 2^115: each one's product with the scales is a denormal number or none."""
    K = K // 128 * 128
    for value, least, exponent in ((0x38, -64, -63), (0x7e, 60, 55)):
        a, b = operand(M, K, "e4m3", scale, 1, 3), operand(N, K, "e4m3", scale, block, 4)
        a[0].view(torch.uint8)[:] = value
        b[0].view(torch.uint8)[:] = value
        if value == 0x7e:
            b[0].view(torch.uint8)[:, 1::2] = value | 0x80
        sa, sb = (torch.full(s.shape, 2.0 ** e, device="cuda").to(scale) for s, e in ((a[1], least), (b[1], exponent)))
        z = A.aal_fp8_matmul(a[0], sa, b[0], sb, out_dtype=out)
        want = 0.0 if value == 0x7e else K * 2.0 ** (least + exponent)
        assert (z.double() == torch.tensor(want).to(out).double().item()).all(), z.flatten()[:4]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_far_blocks_beside_any_others(A, M, N, K):  # noqa: F811
    """Small scales beside large ones, whose products are ordinary, in the same tile as those that are not."""
    for scale in (F32, E8M0):
        for out in (BF16, F32):
            a, b = operand(M, K, "e4m3", scale, 1, 7), operand(N, K, "e4m3", scale, 1, 8)
            g = torch.Generator().manual_seed(9)
            e = torch.randint(-60, 61, (1, a[1].shape[1]), generator=g).float().cuda()
            sa = (a[1].float() * torch.exp2(e)).to(scale)
            sb = (b[1].float() * torch.exp2(-e)).to(scale)
            check(A.aal_fp8_matmul(a[0], sa, b[0], sb, out_dtype=out), (a[0], sa), (b[0], sb), out)
            # no pair of rows in such a block has a product of scales that fp32 holds
            sa[:, 0] = torch.tensor(2.0 ** -75).to(scale)
            sb[:, 0] = torch.tensor(2.0 ** -76).to(scale)
            check(A.aal_fp8_matmul(a[0], sa, b[0], sb, out_dtype=out), (a[0], sa), (b[0], sb), out)


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("block", [1, 128])
def test_negative_scales_and_zeros(A, M, N, K, out, block):  # noqa: F811
    """Scales of either sign, zeros among them, beside others and in blocks that are out of range.  Results below
    2^-126 are rounded to steps of 2^-149, once a block, or of bf16's 2^-133 in the end."""
    a, b = operand(M, K, "e4m3", F32, 1, 11), operand(N, K, "e4m3", F32, block, 12)
    g = torch.Generator("cuda").manual_seed(13)
    for s in (a[1], b[1]):
        s.mul_(torch.randint(-1, 2, s.shape, generator=g, device="cuda"))

    def compare():
        got = A.aal_fp8_matmul(*a, *b, out_dtype=out).double().cpu().numpy()
        host = [t.float().double().cpu().numpy() for t in (*a, *b)]
        want, mag, blocks = H.product(*host), H.magnitude(*host), a[1].shape[1]
        tol = (128 * 2.0 ** -23 + (blocks + 2) * 2.0 ** -24) * mag + blocks * 2.0 ** -149
        if out == BF16:
            tol = tol + 7 * 2.0 ** -13 * mag
            tol = tol + 2.0 ** -8 * (np.abs(want) + tol) + 2.0 ** -134
        assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)

    compare()
    a[1][:, ::2] *= 2.0 ** -70
    b[1][:, ::2] *= 2.0 ** -66
    compare()
    a[1][:, 1::2] = 0
    compare()


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("scale", [F32, E8M0])
def test_scales_that_are_not_numbers(A, M, N, K, out, scale):  # noqa: F811
    """A row's and a column's scale that is NaN (or infinite): theirs are not finite, the others are what they were."""
    a, b = operand(M, K, "e4m3", scale, 1, 14), operand(N, K, "e4m3", scale, 1, 15)
    want = A.aal_fp8_matmul(*a, *b, out_dtype=out)
    for bad in (float("nan"), float("inf")) if scale == F32 else (float("nan"),):
        sa, sb = a[1].float(), b[1].float()
        sa[2, 1], sb[N - 3, 2] = bad, bad
        got = A.aal_fp8_matmul(a[0], sa.to(scale), b[0], sb.to(scale), out_dtype=out)
        there = torch.zeros(M, N, dtype=torch.bool, device="cuda")
        there[2], there[:, N - 3] = True, True
        assert torch.equal(got.isfinite(), ~there)
        tol = 2.0 ** -7 if out == BF16 else 2.0 ** -18  # one bf16 step, or other rounding of the blocks beside it
        assert ((got - want)[~there].abs() <= tol * want[~there].abs() + 2.0 ** -13 * want.abs().max()).all()


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("scale", [F32, E8M0])
@pytest.mark.parametrize("block", [1, 128])
def test_infinite_values(A, M, N, K, out, scale, block):  # noqa: F811
    """e5m2's infinities, in blocks of ordinary scales and of scales out of range: their rows and columns are not finite, the
    others are."""
    a, b = operand(M, K, "e5m2", scale, 1, 16), operand(N, K, "e5m2", scale, block, 17)
    a[0].view(torch.uint8)[3, 200] = 0x7c
    b[0].view(torch.uint8)[N - 5, 3] = 0xfc
    there = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    there[3], there[:, N - 5] = True, True
    for e in (0, -70):
        sa, sb = ((s.float() * 2.0 ** e).to(scale) for s in (a[1], b[1]))
        assert torch.equal(A.aal_fp8_matmul(a[0], sa, b[0], sb, out_dtype=out).isfinite(), ~there)

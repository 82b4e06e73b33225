"""aal_fp8_matmul against the fp64 oracle.

Tolerances, relative to M = sum_k |a b| with the scales.  fp32 results: the values are exact in bf16 and so are
their products in fp32; a block's 128 additions round (or cut) by at most 2^-23 each, the product of the scales by
2^-24, and so does the sum of each block: 128 2^-23 + (blocks + 2) 2^-24 (asked as well where scales are powers of two,
though sums run on from block to block there).  bf16 results: the matrix unit's sums of
8-bit products keep, of each eight neighbours, what lies above 2^-13 of the largest product's power of two, so that each of
eight is off by at most 2^-13 of the largest, the largest itself by nothing: 7 2^-13 of the eight's sum of
|a b| and so of M; rounding to bf16 adds 2^-8 of the value."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as H

pytestmark = pytest.mark.gpu

BF16, F32, E8M0 = torch.bfloat16, torch.float32, torch.float8_e8m0fnu
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_24150_amd as lib
    return lib


def operand(rows, K, fmt, scale, block, seed, behind=0x7f):
    """Values and scales of random numbers; the bytes behind a row's K values are NaN."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, K, generator=g) * (4.0 if fmt == "e4m3" else 50.0)
    q = torch.full((rows, (K + 15) // 16 * 16 + 16), behind, dtype=torch.uint8)
    q[:, :K] = x.to(FP8[fmt]).view(torch.uint8)
    n = rows if block == 1 else (rows + 127) // 128
    nb = (K + 127) // 128
    s = torch.exp2(torch.randint(-9, 3, (n, nb), generator=g).float())
    if scale == F32:
        s = s * (1 + torch.rand(n, nb, generator=g))
    return q.cuda().view(FP8[fmt])[:, :K], s.to(scale).cuda()


def check(out, a, b, dtype):
    host = [t.float().double().cpu().numpy() for t in (*a, *b)]
    want, mag = H.product(*host), H.magnitude(*host)
    tol = (128 * 2.0 ** -23 + (host[1].shape[1] + 2) * 2.0 ** -24) * mag
    if dtype == BF16:
        tol = tol + 7 * 2.0 ** -13 * mag
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    got = out.double().cpu().numpy()
    assert out.dtype == dtype and got.shape == want.shape
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)


SIZES = [(1, 1, 1), (1, 250, 64), (3, 16, 129), (7, 1000, 512), (16, 515, 384), (17, 300, 1000), (33, 129, 257),
         (64, 64, 128), (65, 257, 640), (100, 2050, 130), (127, 255, 127), (128, 256, 128), (129, 257, 272),
         (256, 256, 512), (300, 511, 1024), (515, 130, 4096)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("scale", [F32, E8M0])
def test_sizes(A, M, N, K, scale):
    for i, (block, out) in enumerate(((128, BF16), (1, F32), (128, F32))):
        a, b = operand(M, K, "e4m3", scale, 1, M + i), operand(N, K, "e4m3", scale, block, N + i + 7)
        check(A.aal_fp8_matmul(*a, *b, out_dtype=out), a, b, out)


@pytest.mark.parametrize("fa", ["e4m3", "e5m2"])
@pytest.mark.parametrize("fb", ["e4m3", "e5m2"])
@pytest.mark.parametrize("M,N,K", [(5, 200, 300), (200, 300, 260)])
@pytest.mark.parametrize("scale", [F32, E8M0])
def test_formats_and_blocks(A, fa, fb, M, N, K, scale):
    for ra in (1, 128):
        for rb in (1, 128):
            a, b = operand(M, K, fa, scale, ra, 3), operand(N, K, fb, scale, rb, 4)
            check(A.aal_fp8_matmul(*a, *b, out_dtype=F32), a, b, F32)


@pytest.mark.parametrize("M,N,K", [(4, 300, 500), (150, 300, 500)])
def test_scales_of_any_strides(A, M, N, K):
    a, b = operand(M, K, "e4m3", F32, 1, 1), operand(N, K, "e4m3", F32, 1, 2)
    want = A.aal_fp8_matmul(*a, *b, out_dtype=F32)
    column = lambda s: s.t().contiguous().t()  # noqa: E731
    wide = torch.zeros(N, 3 * b[1].shape[1], device="cuda")[:, ::3]
    wide.copy_(b[1])
    for sa, sb in ((column(a[1]), b[1]), (a[1], column(b[1])), (a[1], wide)):
        assert torch.equal(A.aal_fp8_matmul(a[0], sa, b[0], sb, out_dtype=F32), want)
    one = torch.full((1, 1), 0.5, device="cuda")
    sa = one.expand(a[1].shape)
    got = A.aal_fp8_matmul(a[0], sa, b[0], b[1], out_dtype=F32)
    assert torch.equal(got, A.aal_fp8_matmul(a[0], sa.contiguous(), b[0], b[1], out_dtype=F32))


@pytest.mark.parametrize("M,N", [(4, 300), (150, 300)])
def test_values_at_the_ends(A, M, N):
    """Largest values, zeros, extreme scales; a NaN stays in its own row and column."""
    K = 256
    for scale in (F32, E8M0):
        a, b = operand(M, K, "e4m3", scale, 1, 1), operand(N, K, "e4m3", scale, 128, 2)
        a[0].view(torch.uint8)[:, :7] = 0x7e   # 448
        b[0].view(torch.uint8)[:, :9] = 0xfe   # -448
        a[0].view(torch.uint8)[1] = 0
        check(A.aal_fp8_matmul(*a, *b, out_dtype=F32), a, b, F32)
        tiny = a[1].clone().view(torch.uint8 if scale == E8M0 else F32)
        tiny[2] = 1 if scale == E8M0 else 2.0 ** -126
        big = b[1].clone().view(torch.uint8 if scale == E8M0 else F32)
        big[0] = 247 if scale == E8M0 else 2.0 ** 120
        sa, sb = tiny.view(scale), big.view(scale)
        sa[3:] = sa[3:].float().mul(2.0 ** -110).to(scale)
        sa[:2] = sa[:2].float().mul(2.0 ** -110).to(scale)
        check(A.aal_fp8_matmul(a[0], sa, b[0], sb, out_dtype=F32), (a[0], sa), (b[0], sb), F32)
        a[0].view(torch.uint8)[3, 200] = 0x7f
        b[0].view(torch.uint8)[250, 3] = 0x7f
        got = A.aal_fp8_matmul(*a, *b, out_dtype=F32)
        nan = torch.zeros(M, N, dtype=torch.bool, device="cuda")
        nan[3] = True
        nan[:, 250] = True
        assert torch.equal(got.isnan(), nan)


def test_rows_behind_stay(A):
    """An output in the middle of an array: nothing else of it is written."""
    for M, N, K in ((3, 257, 200), (130, 257, 200), (130, 100, 4000)):
        a, b = operand(M, K, "e4m3", F32, 1, 1), operand(N, K, "e4m3", F32, 128, 2)
        full = torch.full((M * N + 256,), 7.0, device="cuda")
        out = full[128:128 + M * N].view(M, N)
        assert A.aal_fp8_matmul(*a, *b, out=out) is out
        assert (full[:128] == 7).all() and (full[128 + M * N:] == 7).all()
        check(out, a, b, F32)


def test_repeatable_and_on_another_stream(A):
    for M, N, K in ((5, 2000, 1024), (600, 700, 3000)):
        a, b = operand(M, K, "e4m3", E8M0, 1, 1), operand(N, K, "e4m3", E8M0, 128, 2)
        want = A.aal_fp8_matmul(*a, *b, out_dtype=F32)
        torch.cuda.synchronize()
        side = [torch.cuda.Stream() for _ in range(2)]
        got = [A.aal_fp8_matmul(*a, *b, out_dtype=F32, stream=s) for s in side for _ in range(3)]
        torch.cuda.synchronize()
        assert all(torch.equal(g, want) for g in got)


def test_captured(A):
    """Two graphs of one call each, replayed between eager calls on other inputs."""
    for M, N, K in ((3, 1000, 512), (300, 400, 2048)):
        a, b = operand(M, K, "e4m3", F32, 1, 1), operand(N, K, "e4m3", F32, 128, 2)
        other = operand(M, K, "e4m3", F32, 1, 8)
        want, want2 = A.aal_fp8_matmul(*a, *b), A.aal_fp8_matmul(*other, *b)
        torch.cuda.synchronize()
        x, s = torch.zeros_like(a[0].view(torch.uint8)), torch.zeros_like(a[1])
        pitch = torch.zeros(M, (K + 15) // 16 * 16, dtype=torch.uint8, device="cuda")
        x = pitch[:, :K]
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                out = A.aal_fp8_matmul(x.view(torch.float8_e4m3fn), s, *b)
            graphs.append((g, out))
        for _ in range(3):
            for v, w in ((a, want), (other, want2)):
                x.copy_(v[0].view(torch.uint8))
                s.copy_(v[1])
                for g, out in graphs:
                    g.replay()
                A.aal_fp8_matmul(*other, *b)
                torch.cuda.synchronize()
                assert all(torch.equal(out, w) for _, out in graphs)


def test_refusals(A):
    a, b = operand(4, 64, "e4m3", F32, 1, 1), operand(6, 64, "e4m3", F32, 1, 2)
    odd = torch.zeros(4, 65, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    for bad in ((a[0][:, :63], a[1], *b), (a[0].cpu(), a[1], *b), (a[0], a[1].cpu(), *b), (a[0], a[1][:3], *b),
                (a[0], torch.ones(4, 2, device="cuda"), *b), (odd[:, :64], a[1], *b), (odd.flatten()[1:65][None], a[1][:1], *b),
                (a[0].t(), a[1], *b), (a[0][:0], a[1][:0], *b)):
        with pytest.raises(ValueError):
            A.aal_fp8_matmul(*bad)
    short = torch.zeros(4 * 80 - 10, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    with pytest.raises(ValueError):  # the last row's memory ends before its stride
        A.aal_fp8_matmul(short.as_strided((4, 64), (80, 1)), a[1], *b)
    for bad in ((a[0], a[1].to(E8M0), *b), (a[0].float(), a[1], *b), (a[0], a[1].bfloat16(), *b)):
        with pytest.raises(TypeError):
            A.aal_fp8_matmul(*bad)
    with pytest.raises(ValueError):
        A.aal_fp8_matmul(*a, *b, out=torch.empty(4, 7, device="cuda"))
    with pytest.raises(TypeError):
        A.aal_fp8_matmul(*a, *b, out_dtype=torch.float16)

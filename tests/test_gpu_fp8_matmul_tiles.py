"""aal_fp8_matmul at sizes that are cut into tiles of 256 x 256 (bf16 results), in one
piece and in parts of the inner dimension, and the head's gradients at such sizes, against
sums in 64 bits.

Tolerances are those of test_gpu_fp8_matmul.py; tests/test_fp8_plan.py holds how each of these
sizes is cut."""
import pytest
import torch

from test_gpu_fp8_matmul import A, BF16, E8M0, F32, operand  # noqa: F401

pytestmark = pytest.mark.gpu

# two tiles down and 126 across; more tiles than CUs, so that a workgroup takes several; one block; 16 blocks; 8 and 4 parts
SIZES = [(300, 32000, 1000), (2053, 16500, 650), (2100, 4200, 128), (290, 30001, 2000), (300, 4000, 15990), (300, 8001, 7900)]
PARTS = [1, 1, 1, 1, 8, 4]


def spread(q, s):
    rows = torch.arange(q.shape[0], device="cuda") // (1 if s.shape[0] == q.shape[0] else 128)
    return q.float().double() * s.float().double()[rows][:, torch.arange(q.shape[1], device="cuda") // 128]


def check(out, a, b, dtype):
    """test_gpu_fp8_matmul.check, its sums formed by the GPU in 64 bits."""
    x, y = spread(*a), spread(*b)
    want, mag = x @ y.t(), x.abs() @ y.abs().t()
    tol = (128 * 2.0 ** -23 + (a[1].shape[1] + 2) * 2.0 ** -24) * mag
    if dtype == BF16:
        tol = tol + 7 * 2.0 ** -13 * mag
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    assert out.dtype == dtype and out.shape == want.shape
    worst = ((out.double() - want).abs() / tol).max().item()
    assert worst <= 1, worst


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("scale", [F32, E8M0])
@pytest.mark.parametrize("ra", [1, 128])
@pytest.mark.parametrize("rb", [1, 128])
def test_sizes(A, M, N, K, scale, ra, rb):  # noqa: F811
    a, b = operand(M, K, "e4m3", scale, ra, M), operand(N, K, "e4m3", scale, rb, N)
    check(A.aal_fp8_matmul(*a, *b), a, b, BF16)


@pytest.mark.parametrize("fa", ["e4m3", "e5m2"])
@pytest.mark.parametrize("fb", ["e4m3", "e5m2"])
@pytest.mark.parametrize("rb", [1, 128])
@pytest.mark.parametrize("M,N,K", [(300, 32000, 1000), (300, 8001, 7900)])
def test_formats(A, M, N, K, fa, fb, rb):  # noqa: F811
    a, b = operand(M, K, fa, F32, 1, 3), operand(N, K, fb, F32, rb, 4)
    check(A.aal_fp8_matmul(*a, *b), a, b, BF16)


@pytest.mark.parametrize("rb", [1, 128])
def test_repeatable_rows_behind_stay_and_a_graph(A, rb):  # noqa: F811
    for M, N, K in ((2053, 16500, 650), (300, 4000, 15990)):
        a, b = operand(M, K, "e4m3", F32, 1, 1), operand(N, K, "e4m3", F32, rb, 2)
        want = A.aal_fp8_matmul(*a, *b)
        full = torch.full((M * N + 512,), 7.0, dtype=BF16, device="cuda")
        out = full[256:256 + M * N].view(M, N)
        assert A.aal_fp8_matmul(*a, *b, out=out) is out and torch.equal(out, want)
        assert (full[:256] == 7).all() and (full[256 + M * N:] == 7).all()
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        again = A.aal_fp8_matmul(*a, *b, stream=side)
        side.synchronize()
        assert torch.equal(again, want)
        s = a[1].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = A.aal_fp8_matmul(a[0], s, *b)
        for factor in (1.0, 2.0, 0.5):
            s.copy_(a[1] * factor)
            graph.replay()
            A.aal_fp8_matmul(*a, *b)
            torch.cuda.synchronize()
            assert torch.equal(got.float(), want.float() * factor)


@pytest.mark.parametrize("scale", [F32, E8M0])
def test_gradients_in_bf16(A, scale):  # noqa: F811
    """Both gradients of a head at such sizes, the weights' in bf16 and in fp32."""
    rows, D, V = 2100, 4100, 2200
    g = torch.Generator("cuda").manual_seed(2)
    w = torch.randn(V, D, generator=g, device="cuda") * 0.05
    x = torch.randn(rows, D, generator=g, device="cuda").to(BF16)
    grad = (torch.randn(rows, V, generator=g, device="cuda") * 1e-3).to(BF16)
    head = A.aal_fp8_quantize(w, block_rows=128, columns=True, scale_dtype=scale)
    q = A.aal_fp8_quantize(grad, columns=True, scale_dtype=scale)
    t = A.aal_fp8_quantize(x, rows=False, columns=True, scale_dtype=scale)
    for dtype in (BF16, F32):
        out = A.aal_head_logits_bwd(grad, x, head, weight_dtype=dtype)
        check(out["grad_w"], (q["qt"], q["scale_t"]), (t["qt"], t["scale_t"]), dtype)
        check(out["grad_x"], (q["q"], q["scale"]), (head["qt"], head["scale_t"]), BF16)

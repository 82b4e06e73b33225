"""aal_fp8_quantize against the fp64 oracle: scales and values are exact (the
division by a power of two is, and the rounding is to nearest even)."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as H

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_24150_amd as lib
    return lib


def make(rows, cols, dtype, seed, kind="plain"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(3 * torch.randn(rows, cols, generator=g))
    if kind == "zeros":
        x[:, : cols // 2 + 1] = 0
        x[::3] = -0.0
    elif kind == "borders":  # largest values at and around the format's, times powers of two
        top = torch.tensor([448.0, 57344.0, 449.0, 447.0, 57345.0, 2.0 ** -130, 3e38, 2.0 ** -149])
        x = x.clamp(-1, 1) * 2.0 ** -20
        x[:, 0] = top[torch.arange(rows) % 8] * torch.where(torch.arange(rows) < 8, 1.0, 2.0 ** -10)
    elif kind == "halves":  # ties of the rounding: odd multiples of half a step
        x = (torch.randint(-31, 32, (rows, cols), generator=g).float() + 0.5) * 0.5
    elif kind == "special":
        u = torch.rand(rows, cols, generator=g)
        x = torch.where(u < 0.02, float("inf"), torch.where(u < 0.04, float("-inf"), torch.where(u < 0.06, float("nan"), x)))
        x[-1] = float("nan")
    elif kind == "range":
        x = x.sign() * torch.exp2(torch.rand(rows, cols, generator=g) * 200 - 120)
    return x.to(dtype)


def check(r, x, fmt, block, rows=True, columns=False):
    for want, q, s, y in ((rows, "q", "scale", x), (columns, "qt", "scale_t", x.t())):
        if not want:
            assert r[q] is None and r[s] is None
            continue
        oq, os = H.quantize(y.double().cpu().numpy(), fmt, block)
        assert tuple(r[q].shape) == oq.shape and tuple(r[s].shape) == os.shape
        assert r[q].stride(0) % 16 == 0 and r[q].data_ptr() % 16 == 0
        assert np.array_equal(r[s].float().double().cpu().numpy(), os)
        np.testing.assert_array_equal(r[q].float().double().cpu().numpy(), oq)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (7, 130), (17, 127), (128, 128), (129, 257), (200, 515)])
def test_sizes(A, rows, cols, block, fmt, dtype):
    x = make(rows, cols, dtype, rows * 1000 + cols).cuda()
    for kw in (dict(), dict(columns=True), dict(rows=False, columns=True)):
        for scale in (F32, torch.float8_e8m0fnu):
            r = A.aal_fp8_quantize(x, block_rows=block, dtype=FP8[fmt], scale_dtype=scale, **kw)
            check(r, x, fmt, block, **kw)


@pytest.mark.parametrize("kind", ["zeros", "borders", "halves", "special", "range"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_values(A, dtype, block, fmt, kind):
    x = make(150, 300, dtype, 5, kind).cuda()
    check(A.aal_fp8_quantize(x, block_rows=block, dtype=FP8[fmt], columns=True), x, fmt, block, columns=True)


def test_strided_rows_and_bytes_behind(A):
    """Rows at any distance and address; what lies behind an output's rows stays."""
    import ctypes
    from paper_2609_24150_amd import _lib
    full = make(40, 301, BF16, 9).cuda()
    x = full[3:, 1:260]
    check(A.aal_fp8_quantize(x, columns=True), x, "e4m3", 1, columns=True)
    check(A.aal_fp8_quantize(x), x, "e4m3", 1)
    R, Cn = x.shape
    q = torch.full((R, 304), 77, dtype=torch.uint8, device="cuda")
    qt = torch.full((Cn, 64), 77, dtype=torch.uint8, device="cuda")
    s, st = torch.empty(3, R, device="cuda"), torch.empty(1, Cn, device="cuda")
    _lib.check(_lib.lib().aal_fp8_quantize(x.data_ptr(), 0, R, Cn, x.stride(0), 0, 0, 1, q.data_ptr(), 304, s.data_ptr(),
                                           qt.data_ptr(), 64, st.data_ptr(), None), "aal_fp8_quantize")
    torch.cuda.synchronize()
    assert (q[:, Cn:] == 77).all() and (qt[:, R:] == 77).all()
    assert np.array_equal(q[:, :Cn].view(FP8["e4m3"]).float().cpu().numpy(),
                          H.quantize(x.double().cpu().numpy(), "e4m3", 1)[0])


def test_refusals(A):
    x = torch.zeros(4, 8, device="cuda")
    for bad in (x[0], x.t(), x.cpu(), x[:0], x[:, ::2]):
        with pytest.raises(ValueError):
            A.aal_fp8_quantize(bad)
    for kw in (dict(block_rows=2), dict(rows=False)):
        with pytest.raises(ValueError):
            A.aal_fp8_quantize(x, **kw)
    for kw in (dict(dtype=F32), dict(scale_dtype=BF16)):
        with pytest.raises(TypeError):
            A.aal_fp8_quantize(x, **kw)
    with pytest.raises(TypeError):
        A.aal_fp8_quantize(x.double())

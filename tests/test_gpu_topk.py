"""aal_topk_logits against the fp64 oracle: ids and logits are exact (ties go to
the lower id), the remainder to a tolerance.

Tolerance of `rest` = ln sum exp(z / T): a term 2^(z sc - m sc) has a relative
error of at most |z sc| 2^-24 (the rounding of sc) + |z sc - m sc| 2^-24 (the
fused multiply-add) + 2^-23 (exp2), times ln 2 where it is an exponent's;
with |z / T| <= 60 that is under 2e-5, sums and the logarithm add less than
1e-6, and the result's own rounding is 2^-24 |rest|.  So 3e-5 absolute."""
import math

import numpy as np
import pytest
import torch

from oracle import toplist_oracle as T

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
REST_TOL = 3e-5


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_24150_amd as lib
    return lib


def rows_of(kind, rows, V, seed):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, V, generator=g) * 3
    if kind == "ties":
        z = torch.randint(-3, 4, (rows, V), generator=g).float()
    elif kind == "equal":
        z = torch.full((rows, V), -1.25)
    elif kind == "zeros":  # both zeros, which tie, among small values of both signs
        z = torch.randint(-1, 2, (rows, V), generator=g).float() * 0.5
        z = torch.where((z == 0) & (torch.rand(rows, V, generator=g) < 0.5), -0.0, z)
    elif kind == "masked":  # most blocked, some rows wholly
        z = torch.where(torch.rand(rows, V, generator=g) < 0.995, -math.inf, z)
        z[::3] = -math.inf
    elif kind == "rising":
        z = torch.linspace(-20, 20, V).expand(rows, V).contiguous()
    elif kind == "falling":
        z = torch.linspace(20, -20, V).expand(rows, V).contiguous()
    elif kind == "clump":  # the largest side by side
        z[:, V // 3:V // 3 + 600] += 12
    elif kind == "wide":
        z = z * 12
    return z


def check(A, z, k, temperature):
    out = A.aal_topk_logits(z, k, temperature)
    host = z.cpu()
    vals, ids, rest = T.top_logits(host.double().numpy(), k, temperature)
    assert np.array_equal(out["ids"].cpu().numpy(), ids)
    assert torch.equal(out["logits"].cpu().double(), torch.from_numpy(vals))
    got = out["rest"].cpu().double().numpy()
    assert np.array_equal(np.isfinite(got), np.isfinite(rest))
    ok = np.isfinite(rest)
    assert np.array_equal(got[~ok], rest[~ok])
    assert np.abs(got[ok] - rest[ok]).max(initial=0.0) <= REST_TOL


SHAPES = [(1, 1, 1), (3, 7, 7), (5, 64, 64), (4, 513, 512), (40, 1000, 256), (7, 1023, 100), (9, 4097, 33),
          (300, 257, 5), (3, 8191, 512), (2, 33001, 64), (2, 50001, 512), (3, 128256, 64), (2, 151936, 1)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,V,k", SHAPES)
def test_shapes(A, rows, V, k, dtype):
    check(A, rows_of("normal", rows, V, V + k).to(dtype).cuda(), k, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["ties", "equal", "zeros", "masked", "rising", "falling", "clump", "wide"])
@pytest.mark.parametrize("rows,V,k", [(4, 1001, 37), (3, 9000, 300), (2, 40003, 64), (2, 128256, 200)])
def test_distributions(A, kind, rows, V, k, dtype):
    check(A, rows_of(kind, rows, V, 5).to(dtype).cuda(), k, 1.0 if kind != "wide" else 2.0)


@pytest.mark.parametrize("rows", [1, 8, 100, 1300])
def test_row_counts_and_temperature(A, rows):
    check(A, rows_of("normal", rows, 2051, rows).to(BF16).cuda(), 20, 0.7)


def test_leading_dimensions_and_no_rest(A):
    z = rows_of("normal", 24, 500, 3).cuda()
    a = A.aal_topk_logits(z.view(2, 3, 4, 500), 6, rest=False)
    b = A.aal_topk_logits(z, 6)
    assert a["rest"] is None and a["ids"].shape == (2, 3, 4, 6)
    assert torch.equal(a["ids"].view(24, 6), b["ids"]) and torch.equal(a["logits"].view(24, 6), b["logits"])
    assert b["rest"].shape == (24,)


def test_same_bits_every_time(A):
    z = rows_of("ties", 64, 20011, 9).to(BF16).cuda()
    z2 = rows_of("normal", 6, 128256, 9).cuda()
    for x, k in ((z, 128), (z2, 50)):
        first = A.aal_topk_logits(x, k)
        for _ in range(5):
            again = A.aal_topk_logits(x, k)
            for n in first:
                assert torch.equal(first[n], again[n]), n


def test_offsets_past_32_bits(A):
    rows, V = 16800, 128256  # 2.15e9 logits
    z = torch.empty(rows, V, dtype=BF16, device="cuda")
    z.normal_(generator=torch.Generator("cuda").manual_seed(1))
    out = A.aal_topk_logits(z, 8)
    tail = A.aal_topk_logits(z[-40:].contiguous(), 8)
    for n in out:
        assert torch.equal(out[n][-40:], tail[n]), n
    check(A, z[-3:].contiguous(), 8, 1.0)


def test_on_another_stream_and_in_a_graph(A):
    z = rows_of("normal", 6, 128256, 11).to(BF16).cuda()
    want = A.aal_topk_logits(z, 32)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = A.aal_topk_logits(z, 32, stream=s)
    s.synchronize()
    for n in want:
        assert torch.equal(want[n], got[n])
    buf = z.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = A.aal_topk_logits(buf, 32)
    for i in range(3):
        buf.copy_(torch.roll(z, 17 * i, 1))
        graph.replay()
        torch.cuda.synchronize()
        ref = A.aal_topk_logits(buf, 32)
        for n in ref:
            assert torch.equal(cap[n], ref[n]), (i, n)


def test_refusals(A):
    z = torch.zeros(4, 100, device="cuda")
    for k in (0, 101, 513):
        with pytest.raises(ValueError):
            A.aal_topk_logits(z, k)
    with pytest.raises(ValueError):
        A.aal_topk_logits(torch.zeros(100, 4, device="cuda").t(), 3)
    with pytest.raises(ValueError):
        A.aal_topk_logits(torch.zeros(4, 100), 3)
    with pytest.raises(ValueError):
        A.aal_topk_logits(torch.zeros(0, 100, device="cuda"), 3)
    with pytest.raises(TypeError):
        A.aal_topk_logits(z.half(), 3)
    for T_ in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(A.AalError):
            A.aal_topk_logits(z, 3, T_)
    with pytest.raises(A.AalError):
        A.aal_topk_logits(torch.zeros(1001, dtype=BF16, device="cuda")[1:].view(10, 100), 3)  # misaligned


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [300, 5000, 40000])
def test_the_types_lowest_value(A, V, dtype):
    low = torch.finfo(dtype).min
    z = rows_of("normal", 6, V, 13)
    z[0, V // 3:] = low
    z[1] = low
    z[2] = low
    z[2, 7] = 2.0
    z[3, 3:] = -math.inf
    z[4] = low
    z[4, ::2] = -math.inf
    z[5, :2] = low
    check(A, z.to(dtype).cuda(), 50, 1.0)


def test_lists_longer_than_what_is_finite(A):
    # grammars that leave fewer tokens than the list has places, all over the row
    for V in (900, 9000, 130000):
        for n in (0, 1, 63, 64, 65, 300):
            z = torch.full((3, V), -math.inf)
            at = torch.randperm(V, generator=torch.Generator().manual_seed(n))[:n]
            z[:, at] = torch.randn(3, n, generator=torch.Generator().manual_seed(V))
            check(A, z.bfloat16().cuda(), 64, 1.0)
            check(A, z.cuda(), 256, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
def test_more_rows_than_a_launch_holds(A, dtype):
    rows, V, k = (1 << 22) + 9, 9, 2
    z = torch.randn(rows, V, generator=torch.Generator("cuda").manual_seed(5), device="cuda").to(dtype)
    out = A.aal_topk_logits(z, k)
    vals, ids = z.double().sort(dim=1, descending=True, stable=True)
    assert torch.equal(out["ids"].long(), ids[:, :k]) and torch.equal(out["logits"].double(), vals[:, :k])
    assert (out["rest"] - vals[:, k:].logsumexp(1)).abs().max() <= REST_TOL

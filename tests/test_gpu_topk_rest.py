"""The remainder of aal_topk_logits where the list lies far above what is left, against the
fp64 oracle: it is -inf only where no finite logit is left.

Tolerance: an exponent z sc - m sc, with m the largest logit left over, is off by the
roundings of sc and of the fused multiply-add, 2^-24 |z sc| each, and the reference m sc
ln 2 by three roundings of its size; exp2, sums and the logarithm add less than 1e-6.
With |z / T| <= 60 among the logits left over that is 3e-5, and in proportion beyond: 3e-5
max(1, |z / T| / 60)."""
import math

import numpy as np
import pytest
import torch

from oracle import toplist_oracle as T

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_24150_amd as lib
    return lib


def check(A, z, k, temperature):
    out = A.aal_topk_logits(z.cuda(), k, temperature)
    vals, ids, rest = T.top_logits(z.double().numpy(), k, temperature)
    assert np.array_equal(out["ids"].cpu().numpy(), ids)
    assert torch.equal(out["logits"].cpu().double(), torch.from_numpy(vals))
    got = out["rest"].cpu().double().numpy()
    ok = np.isfinite(rest)
    assert np.array_equal(np.isfinite(got), ok), (got, rest)
    assert (np.abs(got - rest)[ok] <= 3e-5 * np.maximum(1.0, np.abs(rest[ok]) / 60)).all(), (got, rest)


def normal(rows, V, seed, width=2.0):
    return torch.randn(rows, V, generator=torch.Generator().manual_seed(seed)) * width


SHAPES = [(40, 1), (300, 8), (1000, 1), (1003, 20), (1500, 200), (3000, 64), (5000, 1), (8000, 20), (9001, 64),
          (20000, 256), (33001, 64), (50001, 512), (128256, 1), (128256, 64)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("gap", [50.0, 88.0, 95.0, 110.0, 300.0])
@pytest.mark.parametrize("V,k", SHAPES)
def test_lists_far_above_the_rest(A, V, k, gap, dtype):
    # row 0: exactly the list lies above; row 1: one more entry; row 2: one entry less; row 3: entries of
    # both kinds between; row 4: the list side by side
    z = normal(5, V, V + k)
    for r, n in enumerate((k, k + 1, k - 1, 2 * k, k)):
        at = torch.randperm(V, generator=torch.Generator().manual_seed(r))[:n] if r < 4 else torch.arange(V // 3, min(V, V // 3 + k))
        z[r, at] += gap
    if V > 3 * k:
        z[3, torch.randperm(V, generator=torch.Generator().manual_seed(9))[:3]] += gap / 2
    for temperature in (1.0, 0.5):
        check(A, z.to(dtype), k, temperature)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V,k", SHAPES)
def test_finite_masks_that_leave_exactly_the_list(A, V, k, dtype):
    for fill in (-1e4, torch.finfo(dtype).min):
        z = torch.full((4, V), fill)
        for r, n in enumerate((k, k + 1, max(1, k - 1), k)):
            at = torch.randperm(V, generator=torch.Generator().manual_seed(r + 3))[:min(n, V)]
            z[r, at] = normal(1, len(at), r)[0]
        z[3, V // 2:] = torch.minimum(z[3, V // 2:], torch.tensor(-math.inf))  # and -inf in half of the last
        check(A, z.to(dtype), k, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V,k", [(2000, 300), (20000, 300), (40001, 64), (128256, 500)])
def test_ties_far_above_and_below(A, V, k, dtype):
    # the list is one value, what is left another: more candidates than any list of them holds
    for n in (k - 1, k, k + 1, V // 2):
        z = torch.full((2, V), -3.0)
        z[0, 100:100 + n] = 120.0
        z[1, V - n:] = 120.0
        z[1, 5] = 119.0
        check(A, z.to(dtype), k, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V,k", SHAPES)
def test_finite_masks_of_every_size(A, V, k, dtype):
    # what fp32 rounds off a product with log2(e) is an exponent of up to 2^-25 of it: hundreds here
    for fill in (-1e8, -2e8, -1e9, -1e10, -3e10, -1e12, -1e20, -1e25, -7e29, -1e31):
        z = torch.full((5, V), fill)
        for r, n in enumerate((k + V // 9, k, 1, k + 1, 0)):
            at = torch.randperm(V, generator=torch.Generator().manual_seed(r + 3))[:min(n, V)]
            z[r, at] = normal(1, len(at), r)[0]
        z[4, V // 2:] = fill / 3
        check(A, z.to(dtype), k, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V,k", [(300, 8), (1003, 20), (3000, 64), (20000, 256), (128256, 64)])
def test_temperatures_near_zero(A, V, k, dtype):
    for temperature in (1e-7, 1e-8, 1e-9, 1e-12, 1e-20, 1e-30, 1e-36):
        for shift in (-9.0, 0.0, 9.0):
            check(A, (normal(3, V, V) + shift).to(dtype), k, temperature)

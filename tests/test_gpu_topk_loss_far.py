"""aal_topk_loss_fwd_bwd where list and remainder are far apart, on the draft's side and on
the target's, and at temperatures near zero, against the fp64 oracle.

Tolerances.  With |z / T| <= 200 an exponent z sc - m sc is off by at most 290 2^-24 (the
rounding of sc) + 290 2^-24 (the fused multiply-add), ln 2 times that is 2.4e-5, exp2 and the sums
add less than 1e-6: every q and p, and sums of them, are within REL = 2.5e-5 of their value, and
a logarithm of one within REL plus 2^-23 of its size (up to 200: 2.4e-5), so 5e-5 = 2 REL.
From these, acceptances are within 2 REL, E within 2 REL K^2, KL (logarithms weighted with
p, which sum to 1; differences of two of them) within 4 REL + 2 REL KL, gradient entries within 6 REL
times the oracle's `bound`, and bf16 ones 2^-8 of their size besides.  Values below 1e-37, which fp32
holds in fewer bits or not at all, are compared to that.  Rows where some q is within 1e-3 of its p are left out of the
comparison of gradients."""
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import toplist_oracle as T

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
REL = 2.5e-5
TINY = 1e-37
WIN, SEQ = 0, 1
WEIGHTS = {"wtv": (1.0, 0.0, 0.0, 0.0), "eal": (0.0, 1.0, 0.0, 0.0), "kl": (0.0, 0.0, 1.0, 0.0),
           "tv": (0.0, 0.0, 0.0, 1.0), "kl+eal": (0.0, 0.1, 1.0, 0.0), "all": (0.5, 0.1, 1.0, 0.3)}


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_24150_amd as lib
    return lib


def check(A, zd, top, ids, rest, K, weights, flags=0, T_d=1.0, T_t=1.0):
    """Windows [N, K, V], tensors on the host."""
    N, _, V = zd.shape
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    host = lambda t: t.detach().cpu().double().numpy()  # noqa: E731
    got = A.aal_topk_loss_fwd_bwd(zd.cuda(), top.cuda(), ids.cuda(), K, rest=cuda(rest), weights=weights, temp_draft=T_d,
                                  temp_target=T_t, flags=flags)
    ref = T.top_loss(host(zd), host(top), ids.numpy(), None if rest is None else host(rest), T_d, T_t, weights, WIN,
                     N, K, K)
    for n in ("accept_tv", "accept_eal"):
        np.testing.assert_allclose(host(got[n]), ref[n], rtol=2 * REL, atol=TINY, err_msg=n)
    for n in ("E_tv", "E_eal"):
        np.testing.assert_allclose(host(got[n]), ref[n], rtol=2 * REL * K * K, atol=TINY, err_msg=n)
    assert np.array_equal(got["xstar"].cpu().numpy(), ref["xstar"])
    kl = ref["terms"][2]
    tol = np.array([2 * REL * K ** 3, 2 * REL * K ** 3, 4 * REL + 2 * REL * abs(kl), 4 * REL])
    assert np.isfinite(host(got["terms"])).all() and math.isfinite(kl), (host(got["terms"]), ref["terms"])
    assert (np.abs(host(got["terms"]) - ref["terms"]) <= tol).all(), (host(got["terms"]), ref["terms"])
    assert abs(got["loss"].item() - ref["loss"]) <= (np.abs(weights) * tol).sum() + 1e-6 * abs(ref["loss"])
    g = host(got["grad"]).reshape(-1, V)
    assert np.isfinite(g).all()
    clear = ref["near"] > 1e-3
    assert clear.any()
    tol = 6 * REL * ref["bound"] + TINY + (2.0 ** -8 * np.abs(ref["grad"]) if got["grad"].dtype == BF16 else 0.0)
    off = np.abs(g - ref["grad"]) > tol
    assert not off[clear].any(), (np.argwhere(off & clear[:, None])[:5], g[off][:5], ref["grad"][off][:5])
    return got, ref


def make(V, k, gap, dtype, seed, N=3, K=3):
    """Lists whose target keeps a fair share in the remainder; draft rows that put all but the list `gap` lower."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(N * K)]).view(N, K, k)
    top = (torch.randn(N, K, k, generator=g) + 2).to(dtype)
    rest = torch.randn(N, K, generator=g) + 2.0
    zd = torch.randn(N, K, V, generator=g) - gap
    zd.scatter_(2, ids, torch.randn(N, K, k, generator=g))
    return zd.to(dtype), top, ids.int(), rest


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("weights", sorted(WEIGHTS))
@pytest.mark.parametrize("gap", [50.0, 80.0, 88.0, 92.0, 100.0, 150.0])
def test_drafts_that_leave_the_remainder_little(A, gap, weights, dtype, flags):
    for V, k in ((90, 64), (700, 8), (4099, 1), (33000, 100)):
        zd, top, ids, rest = make(V, k, gap, dtype, V)
        check(A, zd, top, ids, rest, 3, WEIGHTS[weights], flags)
    zd, top, ids, rest = make(1003, 20, gap / 2, dtype, 5)
    check(A, zd, top, ids, rest, 3, WEIGHTS[weights], flags, T_d=0.5)


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("weights", sorted(WEIGHTS))
@pytest.mark.parametrize("gap", [50.0, 88.0, 120.0])
def test_drafts_that_leave_the_list_little(A, gap, weights, dtype, flags):
    for V, k in ((90, 64), (700, 8), (33000, 100)):
        zd, top, ids, rest = make(V, k, -gap, dtype, V + 1)
        check(A, zd, top, ids, rest, 3, WEIGHTS[weights], flags)


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
@pytest.mark.parametrize("weights", sorted(WEIGHTS))
def test_a_remainder_of_one_entry(A, weights, flags):
    """One finite entry beside the list, where the draft's share of it is near what fp32 holds."""
    for k in (1, 8, 64, 500):
        for gap, more in itertools.product((80.0, 84.0, 86.0, 87.0, 87.3, 87.5, 88.0, 90.0, 103.0), (0.0, 8.0)):
            zd, top, ids, rest = make(900, k, 0.0, F32, k)
            rest = rest + more
            for n in range(3):
                for j in range(3):
                    zd[n, j] = -math.inf
                    zd[n, j, ids[n, j].long()] = 0.0
                    free = next(v for v in range(900) if v not in set(ids[n, j].tolist()))
                    zd[n, j, free] = -gap
            check(A, zd, top, ids, rest, 3, WEIGHTS[weights], flags)


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
@pytest.mark.parametrize("weights", sorted(WEIGHTS))
def test_targets_with_little_or_nearly_all_in_the_remainder(A, weights, flags):
    for k in (1, 8, 64, 500):
        for gap in (60.0, 80.0, 84.0, 85.5, 86.5, 87.0, 87.3, 90.0, 120.0, -60.0, -80.0, -84.0, -87.0, -90.0, -120.0):
            zd, top, ids, rest = make(900, k, 1.0, F32, k + 7)
            top = torch.zeros_like(top)  # all alike: the sum of the list is k
            rest = torch.full_like(rest, -gap)
            check(A, zd, top, ids, rest, 3, WEIGHTS[weights], flags)


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("T_d", [1e-28, 1e-30, 1e-33, 1e-36, 1e-37])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_temperatures_near_zero(A, T_d, sign, dtype, flags):
    # q is 1 at the row's largest logit, listed or not, and 0 elsewhere (two equal ones: a half each)
    for V in (90, 1000, 5003):
        zd, top, ids, rest = make(V, 8, 0.0, dtype, V + 2)
        zd = sign * (1 + zd.abs() * 8)
        zd[0, 0, 3] = zd[0, 0].max()
        listed = ids[1, 1, 2].item()
        zd[1, 1, listed] = zd[1, 1].max() * (2.0 if sign > 0 else 0.5)
        for weights in ("wtv", "eal", "tv"):
            check(A, zd, top, ids, rest, 3, WEIGHTS[weights], flags, T_d=T_d)


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("fill", [-1e8, -2e8, -1e9, -1e10, -3e10, -1e12, -1e20, -1e25, -7e29, -1e31])
def test_finite_masks_of_every_size(A, fill, dtype, flags):
    # what fp32 rounds off a product with log2(e) is an exponent of up to 2^-25 of it: hundreds here
    for V in (300, 1003, 9000, 33001):
        zd, top, ids, rest = make(V, 8, 0.0, dtype, V + 3, N=4)
        g = torch.Generator().manual_seed(V)
        zd = torch.where(torch.rand(zd.shape, generator=g) < 0.9, torch.full_like(zd, fill), zd)
        # a share of the row left on both sides, so that KL is one that fp64 holds
        zd.scatter_(2, ids.long(), torch.randn(ids.shape, generator=g).to(dtype))
        check(A, zd, top, ids, rest, 3, WEIGHTS["all"], flags)
        # all but the list masked, all of the list masked, whole rows, and rows with two fills
        zd[0] = fill
        zd[0].scatter_(1, ids[0].long(), torch.randn(ids[0].shape, generator=g).to(dtype))
        zd[1].scatter_(1, ids[1].long(), fill)
        zd[2] = fill
        zd[3, :, V // 2:] = fill / 3
        zd[3, :, : V // 2] = fill
        for weights in ("wtv", "eal", "tv"):
            check(A, zd, top, ids, rest, 3, WEIGHTS[weights], flags)

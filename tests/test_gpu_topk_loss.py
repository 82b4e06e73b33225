"""aal_topk_loss_fwd_bwd against the fp64 oracle.

Tolerances.  With |z / T| <= 40 an exponent z sc - m sc has an absolute error of
at most 58 2^-24 (the rounding of sc) + 58 2^-24 (the fused multiply-add), ln 2
times that is 4.8e-6, exp2 and the sums add less than 1e-6: every q and p, and
sums of them, are within REL = 1e-5 of their value.  So acceptances are within
2 REL, a window's E (at most K products of K of them) within 2 REL K^2, KL
(sum p |ln p/q| <= 60, and its logarithms' errors of 1e-5 times sum p = 1)
within 7e-4 at worst and REL (1 + KL) in the mean over the differently rounded
entries; the test takes 4 REL (1 + KL).  A gradient entry moves by at most 6
REL times the oracle's `bound` (each of its factors by 2 REL), and a bf16 one
by half an ulp, 2^-8 of its size, besides.  Rows where some q is within 1e-4 of
its p (a sign of q < p that rounding decides) are left out of the comparison
of gradients."""
import math

import numpy as np
import pytest
import torch

from oracle import toplist_oracle as T

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
REL = 1e-5
WIN, SEQ = 0, 1


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_24150_amd as lib
    return lib


def make(B, S, V, k, dtype, seed, cut=False, top_dtype=None, T_t=1.0):
    """Draft logits, and lists whose target resembles the draft."""
    g = torch.Generator().manual_seed(seed)
    zt = torch.randn(B * S, V, generator=g) * 2
    zt[:, torch.randperm(V, generator=g)[:3]] += 4
    zd = (0.8 * zt + torch.randn(B * S, V, generator=g)).to(dtype)
    zt = zt.to(top_dtype or dtype)
    vals, ids, rest = T.top_logits(zt.double().numpy(), k, T_t)
    top, ids = torch.from_numpy(vals).to(zt.dtype), torch.from_numpy(ids).int()
    rest = torch.from_numpy(rest).float()
    if cut:
        n = torch.randint(0, k + 1, (B * S,), generator=g)
        gone = torch.arange(k)[None] >= n[:, None]
        odd = torch.arange(B * S)[:, None] % 3
        top = torch.where(gone & (odd == 0), -math.inf, top.float()).to(zt.dtype)   # by logit,
        ids = torch.where(gone & (odd == 1), -1, ids)                               # by id,
        ids = torch.where(gone & (odd == 2), V + 7, ids).int()                      # by an id past the end
    return zd.view(B, S, V).cuda(), top.view(B, S, k).cuda(), ids.view(B, S, k).cuda(), rest.view(B, S).cuda()


def check(A, zd, top, ids, rest, K, weights, layout, T_d=1.0, T_t=1.0, grad_dtype=None, flags=0, scale=None,
          grad=True, outputs=True):
    B, S, V = zd.shape
    gs = None if scale is None else torch.tensor([scale], device="cuda")
    got = A.aal_topk_loss_fwd_bwd(zd, top, ids, K, rest=rest, weights=weights, temp_draft=T_d, temp_target=T_t,
                                  layout=layout, grad_dtype=grad_dtype, flags=flags, grad_scale=gs, grad=grad,
                                  outputs=outputs)
    host = lambda t: t.detach().cpu().double().numpy()  # noqa: E731
    ref = T.top_loss(host(zd), host(top), ids.cpu().numpy(), None if rest is None else host(rest), T_d, T_t, weights,
                     layout, B, S, K, grad_scale=1.0 if scale is None else scale)
    if outputs:
        for n in ("accept_tv", "accept_eal"):
            np.testing.assert_allclose(host(got[n]), ref[n], rtol=2 * REL, atol=2 * REL * 1e-3, err_msg=n)
        for n in ("E_tv", "E_eal"):
            np.testing.assert_allclose(host(got[n]), ref[n], rtol=2 * REL * K * K, atol=1e-7, err_msg=n)
        assert np.array_equal(got["xstar"].cpu().numpy(), ref["xstar"])
    kl = ref["terms"][2]
    tol = np.array([2 * REL * K * K * K, 2 * REL * K * K * K, 4 * REL * (1 + abs(kl)), 4 * REL])
    if math.isfinite(kl):
        assert (np.abs(host(got["terms"]) - ref["terms"]) <= tol).all(), (host(got["terms"]), ref["terms"])
        assert abs(got["loss"].item() - ref["loss"]) <= (np.abs(weights) * tol).sum() + 1e-6 * abs(ref["loss"])
    else:
        assert got["loss"].item() == ref["loss"] == math.inf
    if not grad:
        assert got["grad"] is None
        return got, ref
    g = host(got["grad"]).reshape(-1, V)
    clear = ref["near"] > 1e-4
    assert clear.mean() > 0.9 or (~clear).sum() <= 2
    tol = 6 * REL * ref["bound"] + 1e-12 + (2.0 ** -8 * np.abs(ref["grad"]) if got["grad"].dtype == BF16 else 0.0)
    off = np.abs(g - ref["grad"]) > tol
    assert not off[clear].any(), (np.argwhere(off & clear[:, None])[:5], g[off][:5], ref["grad"][off][:5])
    return got, ref


WEIGHTS = {"wtv": (1.0, 0.0, 0.0, 0.0), "eal": (0.0, 1.0, 0.0, 0.0), "kl": (0.0, 0.0, 1.0, 0.0),
           "tv": (0.0, 0.0, 0.0, 1.0), "kl+eal": (0.0, 0.1, 1.0, 0.0), "all": (0.5, 0.1, 1.0, 0.3)}


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("weights", sorted(WEIGHTS))
@pytest.mark.parametrize("layout,B,S,K", [(WIN, 6, 4, 4), (SEQ, 2, 13, 5)], ids=["windows", "sequences"])
def test_terms(A, layout, B, S, K, weights, dtype, flags):
    for with_rest, cut in ((True, False), (False, True), (True, True)):
        zd, top, ids, rest = make(B, S, 1000, 17, dtype, 7, cut)
        check(A, zd, top, ids, rest if with_rest else None, K, WEIGHTS[weights], layout, flags=flags)


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("B,S,V,k,K", [
    (1, 1, 1, 1, 1), (2, 2, 3, 3, 2), (3, 1, 9, 2, 1), (2, 3, 65, 64, 3), (1, 64, 300, 5, 64), (5, 7, 1001, 100, 7),
    (3, 8, 2049, 512, 8), (2, 16, 4099, 33, 16), (2, 7, 16032, 50, 7), (1, 5, 33003, 256, 5), (2, 3, 50257, 20, 3),
    (1, 7, 128256, 64, 7), (1, 2, 151936, 10, 2), (1, 2, 262147, 40, 2)])
def test_shapes(A, B, S, V, k, K, dtype, flags):
    zd, top, ids, rest = make(B, S, V, k, dtype, V + k)
    check(A, zd, top, ids, rest, K, WEIGHTS["all"], WIN, flags=flags)
    if S > 1:
        check(A, zd, top, ids, rest, max(1, K - 1), WEIGHTS["all"], SEQ, flags=flags)


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
def test_more_rows_than_run_at_once(A, flags):
    zd, top, ids, rest = make(3, 1500, 130, 12, BF16, 21)
    check(A, zd, top, ids, rest, 6, WEIGHTS["all"], SEQ, flags=flags)
    zd, top, ids, rest = make(900, 7, 130, 12, F32, 22, cut=True)
    check(A, zd, top, ids, None, 7, WEIGHTS["all"], WIN, flags=flags)


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
def test_types_temperatures_scale(A, flags):
    zd, top, ids, rest = make(2, 9, 1003, 31, BF16, 3, top_dtype=F32, T_t=1.3)
    check(A, zd, top, ids, rest, 4, WEIGHTS["all"], SEQ, T_d=0.7, T_t=1.3, grad_dtype=F32, scale=-2.5, flags=flags)
    zd, top, ids, rest = make(2, 9, 1000, 31, F32, 4, top_dtype=BF16, T_t=0.6)
    check(A, zd, top, ids, rest, 4, WEIGHTS["all"], SEQ, T_d=1.4, T_t=0.6, grad_dtype=BF16, scale=3.0, flags=flags)
    check(A, zd, top, ids, rest, 4, WEIGHTS["all"], SEQ, T_t=0.6, grad=False, flags=flags)
    check(A, zd, top, ids, rest, 4, WEIGHTS["wtv"], SEQ, T_t=0.6, outputs=False, flags=flags)


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
def test_rows_without_a_target_and_windows_that_do_not_fit(A, dtype, flags):
    zd, top, ids, rest = make(2, 6, 500, 9, dtype, 5)
    top[0, 2] = -math.inf
    rest[0, 2] = -math.inf
    ids[1, 4] = -1
    rest[1, 4] = -math.inf
    top[1, 0] = -math.inf  # only the remainder left
    zd[0, 2] = -math.inf   # blocked on both sides
    got, _ = check(A, zd, top, ids, rest, 3, WEIGHTS["all"], SEQ, flags=flags)
    assert not got["grad"][0, 2].any() and not got["grad"][1, 4].any()
    assert got["xstar"].view(2, 6)[0, 2] == -1
    got, ref = check(A, zd, top, ids, rest, 7, (0.0, 0.0, 1.0, 0.0), SEQ, flags=flags)  # no window of 7 in 6
    assert got["E_tv"].numel() == 0 and got["terms"][0] == 0
    got, _ = check(A, zd, top, ids, rest, 7, (1.0, 1.0, 0.0, 1.0), SEQ, flags=flags)
    assert got["loss"].item() == 0 and not got["grad"].any()


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
def test_blocked_draft_entries(A, flags):
    # entries blocked on the draft's side: infinite KL where the target wants them, finite gradients
    zd, top, ids, rest = make(3, 3, 700, 8, F32, 6)
    zd[:, :, 100:] = -math.inf
    got, ref = check(A, zd, top, ids, rest, 3, WEIGHTS["wtv"], WIN, flags=flags)
    got = A.aal_topk_loss_fwd_bwd(zd, top, ids, 3, rest=rest, weights=WEIGHTS["kl"], flags=flags)
    assert got["loss"].item() == math.inf and torch.isfinite(got["grad"]).all()
    # everything outside the list blocked: no mass to share the remainder's
    zd = torch.full_like(zd, -math.inf)
    zd.scatter_(2, ids.long(), torch.randn(3, 3, 8, generator=torch.Generator().manual_seed(1)).cuda())
    check(A, zd, top, ids, None, 3, WEIGHTS["all"], WIN, flags=flags)
    got = A.aal_topk_loss_fwd_bwd(zd, top, ids, 3, rest=rest, weights=WEIGHTS["all"], flags=flags)
    assert torch.isfinite(got["grad"]).all()


def test_lists_of_the_whole_vocabulary_give_the_full_objective(A):
    from paper_2609_24150_amd.inputs import make_logits
    V, k = 512, 512
    zd, zt = make_logits("c1", (6, 5, V), F32, seed=3, device="cuda")
    full = A.aal_loss_fwd_bwd(zd, zt, 3, weights=WEIGHTS["all"], layout=SEQ, temp_draft=0.9, temp_target=0.9)
    lst = A.aal_topk_logits(zt, k, 0.9)
    got = A.aal_topk_loss_fwd_bwd(zd, lst["logits"], lst["ids"], 3, rest=lst["rest"], weights=WEIGHTS["all"],
                                  layout=SEQ, temp_draft=0.9, temp_target=0.9)
    for n in ("loss", "terms", "E_tv", "E_eal", "accept_tv", "accept_eal"):
        torch.testing.assert_close(got[n], full[n], rtol=4 * REL, atol=4 * REL)
    assert torch.equal(got["xstar"], full["xstar"])
    torch.testing.assert_close(got["grad"], full["grad"], rtol=4 * REL, atol=1e-6)


def test_gradient_against_differences(A):
    # central differences of the fp32 loss along random directions, for the terms without kinks: the
    # loss has errors of 1e-6, a step of 0.05 curvature errors of its square times a third
    # derivative of order one (the oracle's differences cover the TV terms)
    zd, top, ids, rest = make(2, 6, 400, 12, F32, 8)
    for w in ("kl", "eal", "kl+eal"):
        f = lambda z: A.aal_topk_loss_fwd_bwd(z, top, ids, 3, rest=rest, weights=WEIGHTS[w], layout=SEQ)  # noqa: E731
        g = f(zd)["grad"].double()
        for seed in range(4):
            d = torch.randn(zd.shape, generator=torch.Generator().manual_seed(seed)).cuda()
            h = 0.05
            num = (f(zd + h * d)["loss"].double() - f(zd - h * d)["loss"].double()) / (2 * h)
            assert abs(num.item() - (g * d.double()).sum().item()) < 5e-3


def test_same_bits_every_time(A):
    for layout, K in ((WIN, 7), (SEQ, 5)):
        zd, top, ids, rest = make(40, 7, 4099, 30, BF16, 9)
        call = lambda: A.aal_topk_loss_fwd_bwd(zd, top, ids, K, rest=rest, weights=WEIGHTS["all"], layout=layout)  # noqa: E731
        first = call()
        for _ in range(5):
            again = call()
            for n in first:
                assert torch.equal(first[n], again[n]), n


def test_offsets_past_32_bits(A):
    B, K, V, k = 2400, 7, 128256, 4  # 2.15e9 logits
    zd = torch.empty(B, K, V, dtype=BF16, device="cuda")
    zd.normal_(generator=torch.Generator("cuda").manual_seed(2))
    lst = A.aal_topk_logits(zd, k)
    got = A.aal_topk_loss_fwd_bwd(zd, lst["logits"], lst["ids"], K, rest=lst["rest"], weights=(1.0, 0, 0, 0),
                                  temp_draft=0.8)
    n = 4
    tail = A.aal_topk_loss_fwd_bwd(zd[-n:].contiguous(), lst["logits"][-n:].contiguous(),
                                   lst["ids"][-n:].contiguous(), K, rest=lst["rest"][-n:].contiguous(),
                                   weights=(n / B, 0, 0, 0), temp_draft=0.8)
    torch.testing.assert_close(got["accept_tv"][-n * K:], tail["accept_tv"], rtol=2 * REL, atol=0.0)
    torch.testing.assert_close(got["grad"][-n:].float(), tail["grad"].float(), rtol=2.0 ** -7, atol=0.0)


def test_on_other_streams_and_in_a_graph(A):
    zd, top, ids, rest = make(64, 7, 8000, 20, BF16, 12)
    call = lambda **kw: A.aal_topk_loss_fwd_bwd(zd, top, ids, 7, rest=rest, weights=WEIGHTS["all"], **kw)  # noqa: E731
    want = call()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(3):
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
            outs.append(call(stream=s, flags=A.AAL_FLAG_COOPERATIVE))
    torch.cuda.synchronize()
    for o in outs:
        for n in want:
            assert torch.equal(want[n], o[n]), n
    buf, ws = zd.clone(), torch.empty(A.aal_topk_loss_workspace_bytes(0, 64, 7, 7), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = A.aal_topk_loss_fwd_bwd(buf, top, ids, 7, rest=rest, weights=WEIGHTS["all"], ws=ws)
    for i in range(3):
        buf.copy_(torch.roll(zd, i, 2))
        ws.fill_(0x3c)
        graph.replay()
        torch.cuda.synchronize()
        ref = A.aal_topk_loss_fwd_bwd(buf, top, ids, 7, rest=rest, weights=WEIGHTS["all"])
        for n in ref:
            assert torch.equal(cap[n], ref[n]), (i, n)


def test_refusals(A):
    zd, top, ids, rest = make(2, 3, 100, 5, F32, 1)
    call = lambda z=zd, t=top, i=ids, K=3, **kw: A.aal_topk_loss_fwd_bwd(z, t, i, K, weights=WEIGHTS["kl"], **kw)  # noqa: E731
    call()
    for bad in (dict(t=top[:, :2]), dict(t=top.half()), dict(i=ids.long()), dict(i=ids[..., :4]), dict(K=2),
                dict(z=zd[0]), dict(z=zd.cpu()), dict(z=zd.transpose(1, 2)), dict(rest=rest.double()),
                dict(rest=rest[:1]), dict(t=top.cpu()), dict(t=top.transpose(0, 1))):
        with pytest.raises((ValueError, TypeError)):
            call(**bad)
    for bad in (dict(temp_draft=0.0), dict(temp_target=math.nan), dict(flags=8),
                dict(ws=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(A.AalError):
            call(**bad)
    with pytest.raises(A.AalError):
        A.aal_topk_loss_fwd_bwd(zd, top, ids, 3, weights=(math.inf, 0, 0, 0))
    with pytest.raises(A.AalError):  # longer than the list's bitmap
        A.aal_topk_loss_fwd_bwd(torch.zeros(1, 1, (1 << 19) + 8, device="cuda"), top[:1, :1].contiguous(),
                                ids[:1, :1].contiguous(), 1, weights=WEIGHTS["kl"])


def test_the_longest_vocabulary(A):
    V = 1 << 19
    zd, top, ids, rest = make(1, 2, V, 9, BF16, 2)
    check(A, zd, top, ids, rest, 2, WEIGHTS["all"], WIN)


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
def test_the_types_lowest_value(A, dtype, flags):
    # masks of the lowest finite value: parts of a row, whole rows, whole rows but one entry, and lists
    low = torch.finfo(dtype).min
    for V in (400, 2003):
        zd, top, ids, rest = make(4, 3, V, 8, dtype, V)
        zd[0, :, V // 2:] = low
        zd[1, 0] = low
        zd[1, 1] = low
        zd[1, 1, 5] = 1.0
        top[2, 0, 3:] = low
        top[2, 1] = low
        rest[2, 1] = -math.inf
        top[3, 0] = low  # all mass in the remainder
        check(A, zd, top, ids, rest, 3, WEIGHTS["wtv"], WIN, flags=flags)
        check(A, zd, top, ids, rest, 3, WEIGHTS["eal"], WIN, flags=flags)
        # with KL: where the draft gives wanted entries nothing it is infinite or beyond fp32, so without those rows
        keep = torch.tensor([2, 3], device="cuda")
        check(A, zd[keep].contiguous(), top[keep].contiguous(), ids[keep].contiguous(), rest[keep].contiguous(), 3,
              WEIGHTS["all"], WIN, flags=flags)
    zd = torch.full((1, 2, 300), low, dtype=dtype, device="cuda")
    zd[0, 1, ::2] = -math.inf
    got = A.aal_topk_loss_fwd_bwd(zd, top[:1, :2].contiguous(), ids[:1, :2].clamp(0, 299).contiguous(), 2,
                                  rest=rest[:1, :2].contiguous(), weights=WEIGHTS["wtv"], flags=flags)
    assert torch.isfinite(got["grad"]).all() and math.isfinite(got["loss"].item())


def test_a_poll_that_times_out(A, monkeypatch):
    # the state a time-out leaves, set by the host: every wait ends at once, the loss reads NaN
    zd, top, ids, rest = make(40, 7, 500, 8, F32, 3)
    monkeypatch.setenv("AAL_TEST_PRESET_TIMEOUT", "1")
    got = A.aal_topk_loss_fwd_bwd(zd, top, ids, 7, rest=rest, weights=WEIGHTS["wtv"])
    torch.cuda.synchronize()
    assert math.isnan(got["loss"].item())
    monkeypatch.delenv("AAL_TEST_PRESET_TIMEOUT")
    check(A, zd, top, ids, rest, 7, WEIGHTS["wtv"], WIN)


@pytest.mark.parametrize("V", [600, 4000, 9000, 18000, 33000, 49000, 66000, 100000, 130000, 153000, 160000])
def test_every_size_of_workgroup(A, V):
    # one row length for each number of waves and vectors, whole vectors and ragged, over more than one round
    for v, dtype in ((V, BF16), (V + 3, BF16), (V // 2 // 4 * 4, F32)):
        zd, top, ids, rest = make(1, 3, v, 6, dtype, v)
        n = 300
        zd, top, ids, rest = (t.repeat(n, *([1] * (t.dim() - 1))) for t in (zd, top, ids, rest))
        for weights, layout in ((WEIGHTS["all"], WIN), (WEIGHTS["kl"], SEQ)):
            call = lambda f: A.aal_topk_loss_fwd_bwd(zd, top, ids, 3, rest=rest, weights=weights, layout=layout, flags=f)  # noqa: E731,B023
            got, ref = call(0), call(A.AAL_FLAG_STREAMING)
            torch.testing.assert_close(got["accept_tv"], ref["accept_tv"], rtol=4 * REL, atol=1e-6)
            torch.testing.assert_close(got["loss"], ref["loss"], rtol=1e-4, atol=1e-6)
            scale = ref["grad"].float().abs().amax().item()
            torch.testing.assert_close(got["grad"].float(), ref["grad"].float(), rtol=2.0 ** -7, atol=20 * REL * scale)
            # every copy of a window gets the same gradient (rows of whole vectors: sums in one order)
            if v % (8 if dtype == BF16 else 4) == 0:
                assert torch.equal(got["grad"][0], got["grad"][-1])


@pytest.mark.parametrize("flags", [0, 1], ids=["default", "streaming"])
def test_more_rows_than_a_launch_holds(A, flags):
    """Windows of one row: a row's results do not depend on the others'.  The first rows and
    those around row 2^22 against a call of their own, which the oracle checks."""
    B, V, k = (1 << 22) + 9, 9, 2
    g = torch.Generator("cuda").manual_seed(5)
    zd = torch.randn(B, 1, V, generator=g, device="cuda")
    t = A.aal_topk_logits(zd.view(B, V) + torch.randn(B, V, generator=g, device="cuda"), k)
    top, ids, rest = t["logits"].view(B, 1, k), t["ids"].view(B, 1, k), t["rest"].view(B, 1)
    whole = A.aal_topk_loss_fwd_bwd(
        zd, top, ids, 1, rest=rest, weights=WEIGHTS["all"], layout=WIN, flags=flags,
        grad_scale=torch.tensor([float(B)], device="cuda"))
    for a in (0, (1 << 22) - 31):
        s = slice(a, a + 40)
        check(A, zd[s].clone(), top[s].clone(), ids[s].clone(), rest[s].clone(), 1, WEIGHTS["all"], WIN, flags=flags)
        part = A.aal_topk_loss_fwd_bwd(zd[s].clone(), top[s].clone(), ids[s].clone(), 1, rest=rest[s].clone(),
                                       weights=WEIGHTS["all"], layout=WIN, flags=flags,
                                       grad_scale=torch.tensor([40.0], device="cuda"))
        for n in ("accept_tv", "accept_eal", "xstar"):
            torch.testing.assert_close(whole[n][s], part[n], rtol=4 * REL, atol=4 * REL)
        torch.testing.assert_close(whole["grad"][s], part["grad"], rtol=24 * REL, atol=24 * REL)

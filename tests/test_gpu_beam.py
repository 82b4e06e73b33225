"""aal_beam_select and aal_beam_reorder against the fp64 oracle: choices are
exact, scores and ranks to a tolerance.

Tolerance: totals are formed in 64 bits but for the exponentials of unlisted logits, whose sum is off by at
most 2^-20 of itself (an argument of up to 128 in size rounded by 2^-18, v_exp_f32 and fp32 sums: far
less on average), and the result is rounded to fp32, 2^-24 of it: 2^-20 + 2^-23 |value| (ranks: relative
to the total, whose division by length^penalty >= 1 only shrinks it)."""
import math

import numpy as np
import pytest
import torch

from oracle import beam_oracle as O

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_24150_amd as lib
    return lib


def make(B, W, V, dtype, seed, kind="plain"):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(B, W, V, generator=g) * 3
    scores = -torch.rand(B, W, generator=g).mul(2).cumsum(1)
    if kind == "equal":
        z = torch.full((B, W, V), -1.25)
    elif kind == "same-beams":  # beams alike in every bit: all ties between them
        z = z[:, :1].expand(B, W, V).contiguous()
        scores = torch.full((B, W), -3.0)
    elif kind == "ties":
        z = torch.randint(-2, 3, (B, W, V), generator=g).float()
        z = torch.where((z == 0) & (torch.rand(z.shape, generator=g) < 0.5), -0.0, z)
    elif kind == "masked":  # few allowed, some rows wholly blocked
        z = torch.where(torch.rand(z.shape, generator=g) < 0.99, -math.inf, z)
        z[:, ::3] = -math.inf
    elif kind == "fills":  # masks of the type's lowest value
        z = torch.where(torch.rand(z.shape, generator=g) < 0.9, torch.finfo(dtype).min, z)
    elif kind == "clump":
        z[:, :, V // 3:V // 3 + 700] += 14
    elif kind == "first":  # the first step: one beam alive
        scores[:, 1:] = -math.inf
    elif kind == "dead":
        scores[:] = -math.inf
    elif kind == "far":  # ranks that fp32 does not tell apart
        scores = scores - 3.0e7
    elif kind == "wide":
        z = z * 15
    return z.to(dtype), scores


def check(A, z, scores, n, T=1.0, finished=None, lengths=None, alpha=0.0, eos=-1, pad=0, **kw):
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    out = A.aal_beam_select(dev(z), dev(scores), n, temperature=T, finished=dev(finished), lengths=dev(lengths),
                            length_penalty=alpha, eos=eos, pad=pad, **kw)
    o = O.select(z.double().numpy(), scores.double().numpy(), n, T, None if finished is None else finished.numpy(),
                 None if lengths is None else lengths.numpy(), alpha, eos, pad)
    for k in ("parents", "tokens", "finished", "lengths"):
        if k != "lengths" or lengths is not None:
            assert np.array_equal(out[k].cpu().numpy(), o[k]), k
    for k in ("scores", "rank"):
        got = out[k].double().cpu().numpy()
        assert np.array_equal(np.isinf(got), np.isinf(o[k]))
        fine = np.isfinite(o[k])
        f = np.abs(o[k][fine] / o["scores"][fine])
        assert np.all(np.abs(got[fine] - o[k][fine]) <= 2.0 ** -20 * f + 2.0 ** -23 * np.abs(o[k][fine])), k
    return out


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,W,V,n", [
    (1, 1, 1, 1), (1, 1, 5, 5), (2, 3, 7, 21), (1, 4, 1000, 4), (3, 5, 1001, 10), (2, 2, 2049, 128), (1, 64, 300, 128),
    (5, 8, 4099, 16), (2, 4, 32000, 8), (1, 1, 50001, 1), (1, 3, 50001, 100), (1, 64, 4097, 128)])
def test_sizes(A, B, W, V, n, dtype):
    check(A, *make(B, W, V, dtype, V + n), n)


@pytest.mark.parametrize("kind", ["equal", "same-beams", "ties", "masked", "fills", "clump", "first", "dead", "far", "wide"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,n", [(300, 7), (5003, 16), (20011, 100)])
def test_values(A, dtype, kind, V, n):
    if kind == "far":  # -3e7 - 1: fp32 scores hold multiples of 2
        z, s = make(2, 5, V, dtype, 3, kind)
        check(A, z, s, n)
        return
    check(A, *make(2, 5, V, dtype, 3, kind), n)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("alpha,T", [(0.0, 1.0), (1.0, 0.75), (0.75, 1.25), (-0.5, 1.0)])
def test_ended_beams_and_lengths(A, dtype, alpha, T):
    B, W, V, n = 4, 6, 1003, 12
    z, scores = make(B, W, V, dtype, 11)
    g = torch.Generator().manual_seed(1)
    finished = torch.rand(B, W, generator=g) < 0.4
    finished[0] = True
    scores[1, 2:] = -math.inf
    lengths = torch.randint(1, 40, (B, W), generator=g, dtype=torch.int32)
    z[:, :, 2] = 12.0  # eos among the best
    check(A, z, scores, n, T, finished, lengths, alpha, eos=2, pad=9)
    check(A, z, scores, n, T, finished, None, 0.0, eos=2, pad=-5)
    z[2][finished[2]] = float("nan")  # rows of beams that have ended are not read
    z[1, 2:] = float("nan")
    dev = A.aal_beam_select(z.cuda(), scores.cuda(), n, finished=finished.cuda(), lengths=lengths.cuda())
    assert torch.isfinite(dev["rank"][2]).all()


def test_every_cut(A):
    """Rows cut into parts of every size, the longest among them."""
    for B, W, V, n, dtype in ((40, 8, 16400, 5, BF16), (300, 4, 3000, 3, F32), (1100, 1, 2500, 2, BF16),
                              (1, 64, 70001, 128, F32), (1, 48, 140001, 120, BF16)):
        z, s = make(B, W, V, dtype, 5)
        some = [0] if B == 1 else [0, B // 2, B - 1]
        out = A.aal_beam_select(z.cuda(), s.cuda(), n)
        o = O.select(z[some].double().numpy(), s[some].double().numpy(), n)
        for k in ("parents", "tokens"):
            assert np.array_equal(out[k][some].cpu().numpy(), o[k]), (k, V)


def test_the_longest_rows_and_streams(A):
    z, s = make(1, 2, 1 << 18, BF16, 4)
    want = check(A, z, s, 9)
    zd, sd = z.cuda(), s.cuda()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [A.aal_beam_select(zd, sd, 9, stream=t) for t in streams for _ in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(g[k], want[k]) for g in got for k in want)


@pytest.mark.parametrize("dtype", [BF16, torch.int32, torch.uint8, F32])
@pytest.mark.parametrize("B,W,shape", [(1, 1, ()), (1, 4, (7,)), (3, 5, (2, 9, 16)), (2, 8, (3, 33)), (2, 33, (5, 8)),
                                       (1, 64, (2, 24)), (2, 20, (129,))])
def test_reorder(A, B, W, shape, dtype):
    g = torch.Generator().manual_seed(W)
    state = torch.randint(0, 100, (B, W, *shape), generator=g).to(dtype)
    for n in sorted({W, 1, min(2 * W, 128), 128}):
        parents = torch.randint(-1, W + 1, (B, n), generator=g, dtype=torch.int32)
        if n == W:
            got = state.cuda()
            assert A.aal_beam_reorder([got], parents.cuda())[0] is got
            assert torch.equal(got.cpu(), torch.from_numpy(O.reorder(state.float().numpy(), parents.numpy())).to(dtype))
        before = torch.full((B, n, *shape), 55).to(dtype)
        out = before.cuda()
        A.aal_beam_reorder([state.cuda()], parents.cuda(), out=[out])
        want = O.reorder(state.float().numpy(), parents.numpy(), before.float().numpy())
        assert torch.equal(out.cpu(), torch.from_numpy(want).to(dtype))


def test_reorder_many_views_at_once(A):
    """Caches narrowed to a range of positions, histories and last states of any alignment, in one call; the rest stays."""
    B, W = 3, 6
    g = torch.Generator().manual_seed(2)
    make_ = lambda *s, t=BF16: torch.randint(0, 250, (B, W, *s), generator=g).to(t).cuda()  # noqa: E731
    full = [make_(2, 50, 16) for _ in range(45)] + [make_(50, t=torch.int32), make_(51, t=torch.uint8), make_(3, 7)]
    views = [t[:, :, :, 13:41] for t in full[:45]] + [full[45][:, :, 5:], full[46][:, :, 1:50], full[47][:, :, :, 2:5]]
    parents = torch.tensor([[1, 0, 2, 2, 5, 4], [5, 4, 3, 2, 1, 0], [0, 1, 2, 3, 4, 5]], dtype=torch.int32)
    before = [t.clone() for t in full]
    A.aal_beam_reorder(views, parents.cuda())
    for t, v, b in zip(full, views, before):
        off = v.storage_offset()
        bv = b.as_strided(v.shape, v.stride(), off)
        bv.copy_(bv.clone()[torch.arange(B)[:, None], parents.long()])
        assert torch.equal(t, b)


def test_reorder_in_a_graph(A):
    B, W = 2, 4
    state = torch.arange(B * W * 100, device="cuda").view(B, W, 100)
    parents = torch.zeros(B, W, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(state)
    A.aal_beam_reorder([state], parents, out=[out])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.aal_beam_reorder([state], parents, out=[out])
    for p in ([[3, 2, 1, 0], [0, 0, 1, 1]], [[1, 1, 1, 1], [2, 3, 0, 1]], [[0, 1, 2, 3], [3, 3, 3, 0]]):
        parents.copy_(torch.tensor(p))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), state.cpu()[torch.arange(B)[:, None], torch.tensor(p)])


def test_refusals(A):
    z, s = (t.cuda() for t in make(2, 3, 50, BF16, 1))
    for kw in (dict(z=z[0]), dict(z=z.cpu()), dict(z=z[:, :, ::2]), dict(n=0), dict(n=129), dict(n=151),
               dict(s=s[:, :2]), dict(s=s.cpu()), dict(s=s.double()), dict(finished=torch.zeros(2, 3, device="cuda")),
               dict(lengths=torch.zeros(2, 3, dtype=torch.int64, device="cuda")), dict(ws=torch.empty(10))):
        a = dict(z=z, s=s, n=4)
        a.update(kw)
        with pytest.raises(ValueError):
            A.aal_beam_select(a.pop("z"), a.pop("s"), a.pop("n"), **a)
    with pytest.raises(ValueError):
        A.aal_beam_select(torch.zeros(1, 65, 4, device="cuda"), torch.zeros(1, 65, device="cuda"), 2)
    for kw in (dict(length_penalty=1.0), dict(temperature=0.0), dict(length_penalty=float("nan")),
               dict(ws=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(A.AalError):
            A.aal_beam_select(z, s, 4, **kw)
    p = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    t = torch.zeros(2, 3, 8, 10, device="cuda")
    for args, out in (([t], [t[:, :, :, :5]]), ([t[:1]], None), ([t.cpu()], None), ([t[:, :2]], None), ([t], []),
                      ([t[:, :, ::2, ::2]], None), ([t[:, :1].expand(2, 3, 8, 10)], None),
                      ([t], [torch.zeros(2, 3, 8, 10, dtype=BF16, device="cuda")]), ([t[:, :, :1].expand(2, 3, 4, 10)], None)):
        with pytest.raises(ValueError):
            A.aal_beam_reorder(args, p, out=out)
    for bad in (p.long(), p.cpu(), p[:, :0], p[:, :2]):
        with pytest.raises(ValueError):
            A.aal_beam_reorder([t], bad)
    assert A.aal_beam_reorder([], p) == []

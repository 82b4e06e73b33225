"""Calls of the 8-bit head and of beam search at the edges of what they take:
offsets past 32 bits, the sizes at which a kernel gives way to another, other
streams, two calls at once, captured quantisation, inputs that are not
numbers, and states that share memory.

Products are of values -1, 0 and 1 with scales of powers of two here, whose sums are whole numbers under 2^24 times a
power of two: exact in whatever order they are formed, so results are compared for equality, as choices
and moved bytes are."""
import math

import numpy as np
import pytest
import torch

from oracle import beam_oracle as O

pytestmark = pytest.mark.gpu

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_24150_amd as lib
    yield lib
    torch.cuda.empty_cache()


def signs(rows, K, seed):
    """Values -1, 0, 1, rows at multiples of 16 bytes with NaN behind their ends, and ones as scales."""
    g = torch.Generator("cuda").manual_seed(seed)
    ld = (K + 15) // 16 * 16
    full = torch.full((rows, ld), 0x7f, dtype=torch.uint8, device="cuda")
    pick = torch.randint(0, 3, (rows, K), generator=g, device="cuda", dtype=torch.uint8)
    full[:, :K] = pick.eq(1).to(torch.uint8) * 0x38 + pick.eq(2).to(torch.uint8) * 0xb8  # 1 and -1 in e4m3
    return full.view(E4M3)[:, :K], torch.ones(rows, (K + 127) // 128, device="cuda")


def exact(a, b):
    return a.float() @ b.float().t()


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 257])
@pytest.mark.parametrize("out", [BF16, F32])
def test_products_at_each_number_of_rows(A, M, out):
    """One to many rows, over inner dimensions on both sides of a block and of a part, and odd numbers of columns."""
    for N, K in ((1, 1), (129, 127), (257, 129), (1000, 1025), (63, 4097)):
        (a, sa), (b, sb) = signs(M, K, M), signs(N, K, N)
        z = A.aal_fp8_matmul(a, sa, b, sb, out_dtype=out)
        assert torch.equal(z, exact(a, b).to(out)), (N, K)


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("M,N", [(5, 300), (300, 260)])
def test_products_of_scales_that_bf16_does_not_hold(A, M, N, block):
    """Blocks whose scales are 2^-127 to 2^-101 and their inverses among others, which fp32 holds the products of."""
    K = 128 * 11 + 60
    (a, _), (b, _) = signs(M, K, 5), signs(N, K, 6)
    g = torch.Generator().manual_seed(M)
    nb = (K + 127) // 128
    e = torch.where(torch.rand(nb, generator=g) < 0.5, torch.randint(101, 127, (nb,), generator=g), torch.zeros(nb, dtype=torch.int64))
    e[:2], e[-1], e[4:7] = 0, 126, torch.tensor([127, 0, 127])
    shift = torch.randint(-2, 3, (1 if block == 128 else N, 1), generator=g)
    rows = (N + 127) // 128 if block == 128 else N
    scale = lambda x: (x + 127).clamp(0, 254).to(torch.uint8).view(torch.float8_e8m0fnu).cuda()  # noqa: E731
    sa = scale(-e[None].expand(M, nb) + 0)
    sb = scale((e[None] - 2 * (e[None] > 0) + shift * (e[None] == 0)).expand(rows, nb))
    k = torch.arange(K) // 128
    factor = torch.exp2((-2.0 * (e[None] > 0) + shift * (e[None] == 0)))[:, k].cuda()  # of b's values, 1 or 128 rows alike
    want = a.float() @ (b.float() * factor).t()
    assert torch.equal(A.aal_fp8_matmul(a, sa, b, sb, out_dtype=F32), want)


def test_products_past_32_bits(A):
    """Operands and results whose last entries lie 2^32 bytes behind the first."""
    (a, sa), (b, sb) = signs(40_000, 128, 1), signs(60_001, 128, 2)
    for out in (BF16, F32):  # 4.8 and 9.6 GB
        z = A.aal_fp8_matmul(a, sa, b, sb, out_dtype=out)
        for r in (0, 20_000, 39_900):
            assert torch.equal(z[r:r + 100], exact(a[r:r + 100], b).to(out))
        del z
    del a, b
    torch.cuda.empty_cache()
    b, sb = signs(70_000, 65_600, 3)  # 4.6 GB
    for M in (1, 300):
        a, sa = signs(M, 65_600, 4)
        for out in (BF16, F32):
            z = A.aal_fp8_matmul(a, sa, b, sb, out_dtype=out)
            y = A.aal_fp8_matmul(b, sb, a, sa, out_dtype=out)
            for r in (0, 40_000, 69_900):
                want = exact(a, b[r:r + 100]).to(out)
                assert torch.equal(z[:, r:r + 100], want) and torch.equal(y[r:r + 100], want.t())


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantisation_past_32_bits(A, block_rows):
    """Blocks of the last rows and columns, against those of a copy of them."""
    R, C = 33_000, 131_201  # 4.3e9 values
    x = torch.empty(R, C, dtype=BF16, device="cuda")
    for r in range(0, R, 1000):
        x[r:r + 1000].normal_(generator=torch.Generator("cuda").manual_seed(r))
    q = A.aal_fp8_quantize(x, block_rows=block_rows, columns=True)
    for r in (0, 16_384, 32_896):
        for c in (0, 131_072):
            part = A.aal_fp8_quantize(x[r:r + 128, c:c + 256].contiguous(), block_rows=block_rows, columns=True)
            rows, cols = part["q"].shape
            same = lambda u, v: torch.equal(u.view(torch.uint8), v.view(torch.uint8))  # noqa: E731
            assert same(q["q"][r:r + rows, c:c + cols].contiguous(), part["q"].contiguous())
            assert same(q["qt"][c:c + cols, r:r + rows].contiguous(), part["qt"].contiguous())
            rs, cs = part["scale"].shape
            assert torch.equal(q["scale"][r // block_rows:r // block_rows + rs, c // 128:c // 128 + cs], part["scale"])
            rs, cs = part["scale_t"].shape
            assert torch.equal(q["scale_t"][c // block_rows:c // block_rows + rs, r // 128:r // 128 + cs], part["scale_t"])


@pytest.mark.parametrize("B,W,V", [(1, 1, 12_001), (1, 2, 50_001), (1, 3, 20_000), (1, 8, 64_001), (2, 4, 32_000), (9, 5, 2_049),
                                   (1, 30, 16_385), (2, 32, 16_384), (3, 20, 33_001)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_selection_from_rows_cut_in_any_way(A, B, W, V, dtype):
    """Few and many parts, of one to eight vectors a thread, from one choice to 128; flat rows and clustered ones."""
    g = torch.Generator().manual_seed(V)
    s = -torch.rand(B, W, generator=g).cumsum(1)
    for i, n in enumerate((1, 9, 64, 65, 128)):
        z = torch.randn(B, W, V, generator=g).mul(0.3 if i % 2 else 3).to(dtype)
        out = A.aal_beam_select(z.cuda(), s.cuda(), n)
        o = O.select(z.double().numpy(), s.double().numpy(), n)
        for k in ("parents", "tokens"):
            assert np.array_equal(out[k].cpu().numpy(), o[k]), (k, n)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_selection_past_32_bits(A, dtype):
    B, W, V, n = (2_200, 8, 128_257, 8) if dtype == BF16 else (1_100, 8, 128_257, 8)  # 4.5 GB
    z = torch.empty(B, W, V, dtype=dtype, device="cuda")
    for b in range(0, B, 100):
        z[b:b + 100].normal_(generator=torch.Generator("cuda").manual_seed(b))
    s = -torch.rand(B, W, generator=torch.Generator().manual_seed(0)).cumsum(1)
    out = A.aal_beam_select(z, s.cuda(), n)
    some = [0, B // 2, B - 1]
    o = O.select(z[some].double().cpu().numpy(), s[some].double().numpy(), n)
    for k in ("parents", "tokens"):
        assert np.array_equal(out[k][some].cpu().numpy(), o[k]), k


def test_reordering_past_32_bits(A):
    B, W, L = 2, 3, 800_000_008  # 4.8 GB
    state = torch.empty(B, W, L, dtype=torch.uint8, device="cuda")
    for i, t in enumerate(state.view(-1, L)):
        t.random_(0, 256, generator=torch.Generator("cuda").manual_seed(i))
    parents = torch.tensor([[2, 0, 0], [1, 2, 0]], dtype=torch.int32, device="cuda")
    out = torch.empty_like(state)
    A.aal_beam_reorder([state], parents, out=[out])
    for b in range(B):
        for j, k in enumerate(parents[b].tolist()):
            assert torch.equal(out[b, j], state[b, k])
    A.aal_beam_reorder([state], parents)
    assert torch.equal(state, out)


def test_other_streams(A):
    """Inputs made on a stream of their own behind other work, some not contiguous: a call for that stream waits for
    them, whatever stream is current, the copies that it makes included."""
    side = torch.cuda.Stream()
    D, V, rows = 192, 801, 256
    g = torch.Generator("cuda").manual_seed(1)
    w = torch.randn(V, D, generator=g, device="cuda")
    x0 = torch.randn(2, D, rows // 2, generator=g, device="cuda", dtype=F32)
    g0 = torch.randn(2, V, rows // 2, generator=g, device="cuda", dtype=F32)
    work = torch.randn(6000, 6000, device="cuda")
    head = A.aal_fp8_quantize(w, block_rows=128, columns=True)
    want_z = A.aal_head_logits(x0.transpose(1, 2), head)
    want = A.aal_head_logits_bwd(g0.transpose(1, 2), x0.transpose(1, 2), head)
    x, gr = torch.zeros_like(x0), torch.zeros_like(g0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(4):
            work @ work
        x.copy_(x0)
        gr.copy_(g0)
    z = A.aal_head_logits(x.transpose(1, 2), head, stream=side)
    r = A.aal_head_logits_bwd(gr.transpose(1, 2), x.transpose(1, 2), head, stream=side)
    q = A.aal_fp8_quantize(x[0], columns=True, stream=side)
    state = torch.arange(12, device="cuda").view(1, 3, 4)
    torch.cuda.current_stream().wait_stream(side)
    A.aal_beam_reorder([state], torch.tensor([[2, 2, 0]], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(z, want_z) and all(torch.equal(r[k], want[k]) for k in want)
    ref = A.aal_fp8_quantize(x0[0], columns=True)
    assert all(torch.equal(q[k].float(), ref[k].float()) for k in q)
    assert state[0, :, 0].tolist() == [8, 8, 0]


def test_two_calls_at_once(A):
    """Products and selections on two streams, each with a workspace of its own."""
    (a, sa), (b, sb) = signs(16, 8192, 1), signs(5000, 8192, 2)
    want = exact(a, b)
    g = torch.Generator("cuda").manual_seed(3)
    z, s = torch.randn(4, 8, 30_001, generator=g, device="cuda"), torch.zeros(4, 8, device="cuda")
    first = A.aal_beam_select(z, s, 8)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [(A.aal_fp8_matmul(a, sa, b, sb, out_dtype=F32, stream=t), A.aal_beam_select(z, s, 8, stream=t))
           for _ in range(4) for t in streams]
    torch.cuda.synchronize()
    for c, r in got:
        assert torch.equal(c, want) and all(torch.equal(r[k], first[k]) for k in r)


def test_quantisation_in_a_graph(A):
    x = torch.zeros(300, 1000, dtype=BF16, device="cuda")
    A.aal_fp8_quantize(x, block_rows=128, columns=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = A.aal_fp8_quantize(x, block_rows=128, columns=True)
    for seed in range(4):
        x.normal_(generator=torch.Generator("cuda").manual_seed(seed))
        if seed == 2:
            x[:] = 0
        graph.replay()
        want = A.aal_fp8_quantize(x, block_rows=128, columns=True)
        torch.cuda.synchronize()
        assert all(torch.equal(out[k].float(), want[k].float()) for k in want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,n", [(300, 7), (5003, 128), (20_011, 100)])
def test_logits_that_are_not_numbers(A, dtype, V, n):
    """Requests with NaN and infinities end in existing beams and tokens, those beside them in the right ones."""
    B, W = 9, 4
    g = torch.Generator().manual_seed(V)
    z = torch.randn(B, W, V, generator=g)
    s = -torch.rand(B, W, generator=g).cumsum(1)
    z[1, 1, 5] = math.nan
    z[2] = math.nan
    z[3, :, ::2] = math.nan
    z[4] = torch.where(torch.rand(W, V, generator=g) < 0.5, math.nan, 0.0)
    z[5, 2] = math.inf
    z[6, :, 1::3] = -math.nan
    s[7, 2] = math.nan
    z[7] = 1.0
    out = A.aal_beam_select(z.to(dtype).cuda(), s.cuda(), n, pad=V + 3)
    parents, tokens = out["parents"].cpu(), out["tokens"].cpu()
    assert ((parents >= -1) & (parents < W)).all()
    assert (((tokens >= 0) & (tokens < V)) | (tokens == V + 3)).all()
    fine = [0, 8]
    o = O.select(z[fine].to(dtype).double().numpy(), s[fine].double().numpy(), n, pad=V + 3)
    assert np.array_equal(parents[fine].numpy(), o["parents"]) and np.array_equal(tokens[fine].numpy(), o["tokens"])


def test_states_that_share_memory(A):
    B, W, L = 2, 4, 48
    p = torch.tensor([[1, 0, 3, 3], [0, 1, 1, 2]], dtype=torch.int32, device="cuda")
    t = torch.zeros(B, W, 2, L, 8, device="cuda")
    u = torch.zeros_like(t)
    for states, out in (([t, t], None), ([t, t[:, :, :1]], None), ([t[:, :, :, :20], t[:, :, :, 19:]], None),
                        ([u, t, u.view(torch.int32)], None), ([t], [t]), ([t], [t.clone(), t][1:]), ([t, u], [u, t]),
                        ([t, t], [u, u]), ([t[:, :, 0], t[:, :, 1]], [u[:, :, 0], u[:, :, 0]])):
        with pytest.raises(ValueError):
            A.aal_beam_reorder(states, p, out=out)
    # the same state read twice, and pieces of one array that do not meet
    t.copy_(torch.arange(t.numel(), device="cuda").view(t.shape))
    want = O.reorder(t.double().cpu().numpy(), p.cpu().numpy())
    v = torch.zeros_like(t)
    A.aal_beam_reorder([t, t], p, out=[u, v])
    assert np.array_equal(u.double().cpu().numpy(), want) and torch.equal(u, v)
    A.aal_beam_reorder([t[:, :, 0], t[:, :, 1, :20], t[:, :, 1, 20:]], p)
    assert torch.equal(t, u)


def test_states_without_bytes(A):
    """A cache of no positions yet, among others, into other buffers and in place."""
    p = torch.tensor([[1, 0, 1]], dtype=torch.int32, device="cuda")
    full = torch.arange(6, device="cuda").view(1, 2, 3)
    empty, out = torch.zeros(1, 2, 0, 8, device="cuda"), torch.zeros(1, 3, 3, dtype=torch.int64, device="cuda")
    A.aal_beam_reorder([empty, full], p, out=[torch.zeros(1, 3, 0, 8, device="cuda"), out])
    assert out.tolist() == [[[3, 4, 5], [0, 1, 2], [3, 4, 5]]]
    A.aal_beam_reorder([empty, full], p[:, :2].contiguous())
    assert full.tolist() == [[[3, 4, 5], [0, 1, 2]]]
    assert A.aal_beam_reorder([empty], p[:, :2].contiguous())[0] is empty


@pytest.mark.parametrize("count", [1, 7, 8, 9, 40, 41, 49, 130])
def test_any_number_of_states(A, count):
    p = torch.tensor([[1, 0, 1], [2, 1, 0]], dtype=torch.int32, device="cuda")
    g = torch.Generator("cuda").manual_seed(count)
    states = [torch.randint(0, 99, (2, 3, 3 + i % 5), generator=g, device="cuda", dtype=(torch.uint8, torch.int32, torch.int64)[i % 3])
              for i in range(count)]
    want = [s[torch.arange(2, device="cuda")[:, None], p.long()] for s in states]
    A.aal_beam_reorder(states, p)
    assert all(torch.equal(s, w) for s, w in zip(states, want))


@pytest.mark.parametrize("W", [2, 5, 12, 20, 40])
def test_pieces_at_any_address(A, W):
    """Segments of 1 to 70 bytes that start anywhere, several of them a slot, in place and from one alignment to another."""
    g = torch.Generator("cuda").manual_seed(W)
    p = torch.randint(0, W, (2, W), generator=g, device="cuda", dtype=torch.int32)
    make = lambda: torch.randint(0, 256, (2, W, 3, 90), generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    sizes = [(i % 17, n) for i, n in enumerate((*range(1, 40), 47, 48, 49, 63, 64, 65, 70))]
    full, other = [make() for _ in sizes], [make() for _ in sizes]
    rows = torch.arange(2, device="cuda")[:, None]
    want, moved = [f.clone() for f in full], [o.clone() for o in other]
    for (at, n), f, w, m in zip(sizes, full, want, moved):
        m[..., 3:3 + n] = f[..., at:at + n][rows, p.long()]
        w[..., at:at + n] = m[..., 3:3 + n]
    views = [f[..., at:at + n] for (at, n), f in zip(sizes, full)]
    A.aal_beam_reorder(views, p, out=[o[..., 3:3 + n] for (_, n), o in zip(sizes, other)])
    assert all(torch.equal(o, m) for o, m in zip(other, moved))
    A.aal_beam_reorder(views, p)
    assert all(torch.equal(f, w) for f, w in zip(full, want))


@pytest.mark.parametrize("W", [1, 2, 4, 7, 9])
def test_large_states_in_place(A, W):
    """More pieces than are looked at one by one, requests that stay whole among others, ends of segments too."""
    B, L = 5, 1 << 20
    g = torch.Generator("cuda").manual_seed(W)
    state = torch.randint(0, 1 << 30, (B, W, 4, L + 7), generator=g, device="cuda", dtype=torch.int32).view(torch.uint8)
    p = torch.randint(-1, W + 1, (B, W), generator=g, device="cuda", dtype=torch.int32)
    p[1] = torch.arange(W)
    p[3] = -1
    view = state[..., 3:-2]
    before = state.clone()
    A.aal_beam_reorder([view], p)
    take = torch.where((p >= 0) & (p < W), p, torch.arange(W, dtype=torch.int32, device="cuda")).long()
    for b in range(B):
        for j in range(W):
            assert torch.equal(state[b, j, :, 3:-2], before[b, take[b, j], :, 3:-2])
    assert torch.equal(state[..., :3], before[..., :3]) and torch.equal(state[..., -2:], before[..., -2:])

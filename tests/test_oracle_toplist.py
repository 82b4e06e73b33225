"""Pins of the oracle of the top-logits operators (CPU): sorting, closed forms,
central differences of the losses, and the full-vocabulary oracle where a list
holds the whole vocabulary."""
import math

import numpy as np
import pytest

import oracle as O
from oracle import toplist_oracle as T


def test_top_logits_against_python_sorting():
    rng = np.random.default_rng(1)
    z = rng.integers(-3, 4, (6, 41)).astype(np.float64)
    z[1] = 0.0
    z[1, ::2] = -0.0
    z[2, 5:] = -math.inf
    z[3] = -math.inf
    vals, ids, rest = T.top_logits(z, 9, 0.7)
    for r in range(6):
        order = sorted(range(41), key=lambda v: (-(z[r, v] + 0.0), v))
        assert ids[r].tolist() == order[:9]
        left = [math.exp(z[r, v] / 0.7) for v in order[9:]]
        if sum(left) > 0:
            assert rest[r] == pytest.approx(math.log(sum(left)), rel=1e-13)
        else:
            assert rest[r] == -math.inf


@pytest.mark.parametrize("layout,B,S,K", [(0, 4, 3, 3), (1, 2, 7, 3), (1, 1, 2, 3)])
@pytest.mark.parametrize("weights", [(1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (0.5, 0.1, 1, 0.3)])
def test_lists_of_the_whole_vocabulary_are_the_full_objective(layout, B, S, K, weights):
    rng = np.random.default_rng(2)
    R, V = B * S, 13
    zd, zt = rng.normal(0, 2, (R, V)), rng.normal(0, 2, (R, V))
    ref = O.combined_loss(zd, zt, 0.8, 1.2, weights, layout, B, S, K)
    vals, ids, rest = T.top_logits(zt, V, 1.2)
    assert (rest == -math.inf).all()
    shuffle = rng.permutation(V)
    for tail in (None, rest):
        got = T.top_loss(zd, vals[:, shuffle], ids[:, shuffle], tail, 0.8, 1.2, weights, layout, B, S, K)
        used = np.array(weights) != 0
        np.testing.assert_allclose(got["terms"][used], ref["terms"][used], rtol=1e-12)
        np.testing.assert_allclose(got["loss"], ref["loss"], rtol=1e-12)
        np.testing.assert_allclose(got["accept_tv"], ref["a_tv"], rtol=1e-12)
        np.testing.assert_allclose(got["accept_eal"], ref["a_eal"], rtol=1e-12)
        np.testing.assert_allclose(got["grad"], ref["grad"], atol=1e-14)
        assert (got["xstar"] == ref["xstar"]).all()


@pytest.mark.parametrize("with_rest", [False, True])
@pytest.mark.parametrize("weights", [(1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (0.5, 0.1, 1, 0.3)])
def test_gradient_against_differences(weights, with_rest):
    rng = np.random.default_rng(3)
    B, S, K, V, k = 2, 5, 3, 11, 4
    zd, zt = rng.normal(0, 1.5, (B * S, V)), rng.normal(0, 1.5, (B * S, V))
    vals, ids, rest = T.top_logits(zt, k, 0.9)
    ids[1, 2], vals[2, 1], ids[3, 0] = -1, -math.inf, V + 5  # padding of all kinds
    vals[4] = -math.inf
    if with_rest:
        rest[4] = -math.inf  # row 4 has no target
    tail = rest if with_rest else None
    f = lambda z: T.top_loss(z, vals, ids, tail, 0.7, 0.9, weights, 1, B, S, K)  # noqa: E731
    got = f(zd)
    assert got["near"].min() > 1e-3  # no kink within a step
    assert (got["grad"][4] == 0).all() and got["xstar"][4] == -1 and got["accept_tv"][4] == 0
    h = 1e-6
    for r in range(B * S):
        for v in range(V):
            up, dn = zd.copy(), zd.copy()
            up[r, v] += h
            dn[r, v] -= h
            num = (f(up)["loss"] - f(dn)["loss"]) / (2 * h)
            assert abs(num - got["grad"][r, v]) < 1e-8, (r, v)


def test_masses_by_hand():
    # p = (1/2, 1/4) and 1/4 left over, q = (1/4, 1/4, 1/2): min sums 1/4 + 1/4 + 1/4
    got = T.top_loss(np.log([[1.0, 1.0, 1.0, 1.0]]), np.log([[2.0, 1.0]]), [[2, 0]], np.log([1.0]), 1.0, 1.0,
                     (0, 0, 1, 1), 0, 1, 1, 1)
    assert got["accept_tv"][0] == pytest.approx(0.75)
    assert got["kl"][0] == pytest.approx(0.5 * math.log(2) + 0.25 * math.log(0.5))
    assert got["xstar"][0] == 2 and got["accept_eal"][0] == pytest.approx(0.25)


def test_processing_by_hand_and_differences():
    V = 40
    rules = dict(tokens=[3, 3, 5, 3, 39, 77, -2], hist_start=[0, 2], hist_len=[5, 9], prompt_len=[1, 0],
                 repetition=[2.0, 1.5], frequency=[0.25, 0.0], presence=[0.5, 1.0], bias_offsets=[0, 2, 3],
                 bias_ids=[5, 5, 1], bias_values=[9.0, -4.0, 2.0], mask=[[-1, 0xFF & ~2]], mask_row=[0, -1])
    z = np.zeros((2, V))
    z[:, 3], z[:, 5], z[:, 39], z[:, 33] = 4.0, 3.0, -1.0, math.nan
    out = T.process_logits(z, rules)
    assert out[0, 3] == 4.0 / 2 - 0.25 * 2 - 0.5          # twice generated, once in the prompt
    assert out[0, 5] == (3.0 - 4.0) * 2 - 0.25 - 0.5      # the later bias, then the penalties
    assert out[0, 39] == -1.0 * 2 - 0.25 - 0.5
    assert out[0, 33] == -math.inf and out[0, 34] == 0.0  # blocked whatever it held
    assert out[1, 3] == 4.0 / 1.5 - 1.0 and out[1, 1] == 2.0
    z[:, 33] = 0.5
    g = np.random.default_rng(4).normal(size=z.shape)
    d = T.process_logits_bwd(g, z, rules)
    h = 1e-6
    for r in range(2):
        for v in range(V):
            up, dn = z.copy(), z.copy()
            up[r, v] += h
            dn[r, v] -= h
            with np.errstate(invalid="ignore"):
                num = (T.process_logits(up, rules)[r, v] - T.process_logits(dn, rules)[r, v]) / (2 * h) * g[r, v]
            if np.isnan(num):
                num = 0.0  # -inf on both sides
            if z[r, v] != 0 or v not in (3, 5, 39):
                assert abs(num - d[r, v]) < 1e-8, (r, v)

"""Pins of the fp64 oracles of the 8-bit head and of beam search: hand-computed
cases, brute force and torch's own 8-bit casts."""
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import beam_oracle as O
from oracle import head_oracle as H

FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_rounding_against_every_value_of_the_format(fmt):
    all_ = torch.arange(256, dtype=torch.uint8).view(FP8[fmt]).double().numpy()
    fine = np.sort(np.unique(all_[np.isfinite(all_)]))
    np.testing.assert_array_equal(H.round_to(fine, fmt), fine)
    assert fine.max() == H.FORMATS[fmt][2]
    mid = (fine[1:] + fine[:-1]) / 2  # ties, and what lies beside them
    for x in (mid, mid * (1 + 1e-9), mid * (1 - 1e-9)):
        near = np.abs(x[:, None] - fine[None]).min(1)
        np.testing.assert_array_equal(np.abs(H.round_to(x, fmt) - x), near)
    np.testing.assert_array_equal(H.round_to(mid, fmt), torch.tensor(mid, dtype=torch.float32).to(FP8[fmt]).double().numpy())
    assert np.isnan(H.round_to(np.array([np.nan]), fmt))[0]
    assert np.isnan(H.round_to(np.array([np.inf]), "e4m3"))[0] and H.round_to(np.array([-np.inf]), "e5m2")[0] == -np.inf


def test_scales_by_hand():
    x = np.zeros((3, 200))
    x[0, 0], x[0, 199], x[1, 5], x[2, 130] = 448.0, 449.0, np.inf, 2.0 ** -140
    q, s = H.quantize(x, "e4m3", 1)
    np.testing.assert_array_equal(s, [[1, 2], [1, 1], [1, 2.0 ** -126]])
    assert q[0, 0] == 448 and q[0, 199] == 224 and np.isnan(q[1, 5])
    q, s = H.quantize(x, "e5m2", 128)
    assert s.shape == (1, 2) and s[0, 0] == 2.0 ** -7 and q[0, 0] == 57344


def test_products_by_loops():
    r = np.random.default_rng(0)
    a, b = r.integers(-8, 9, (3, 300)).astype(float), r.integers(-8, 9, (130, 300)).astype(float)
    sa, sb = r.random((3, 3)), r.random((2, 3))
    got = H.product(a, sa, b, sb)
    for m, n in ((0, 0), (2, 129), (1, 127), (1, 128)):
        want = sum(sa[m, k // 128] * sb[n // 128, k // 128] * a[m, k] * b[n, k] for k in range(300))
        assert abs(got[m, n] - want) < 1e-9
    assert (H.magnitude(a, sa, b, sb) >= np.abs(got)).all()


@pytest.mark.parametrize("alpha", [0.0, 1.0])
def test_selection_against_all_candidates(alpha):
    r = np.random.default_rng(1)
    B, W, V, n = 2, 3, 7, 9
    z, scores = r.normal(size=(B, W, V)), -r.random((B, W)).cumsum(1)
    finished = np.array([[0, 1, 0], [1, 1, 1]], bool)
    lengths = r.integers(1, 9, (B, W))
    z[0, 2, 3] = -math.inf
    o = O.select(z, scores, n, 0.5, finished, lengths, alpha, eos=4, pad=6)
    for b in range(B):
        cands = []
        for w, v in itertools.product(range(W), range(V)):
            if finished[b, w]:
                if v == 0:
                    cands.append((scores[b, w] / lengths[b, w] ** alpha, w, 6, scores[b, w], True, lengths[b, w]))
            elif z[b, w, v] > -math.inf:
                p = np.exp(z[b, w] / 0.5)
                t = scores[b, w] + math.log(p[v] / p.sum())
                cands.append((t / (lengths[b, w] + 1) ** alpha, w, v, t, v == 4, lengths[b, w] + 1))
        cands.sort(key=lambda c: -c[0])
        for j in range(n):
            if j < len(cands):
                c = cands[j]
                assert abs(o["rank"][b, j] - c[0]) < 1e-12 and abs(o["scores"][b, j] - c[3]) < 1e-12
                assert (o["parents"][b, j], o["tokens"][b, j], o["finished"][b, j], o["lengths"][b, j]) == (c[1], c[2], c[4], c[5])
            else:
                assert o["scores"][b, j] == -math.inf and o["parents"][b, j] == -1 and o["tokens"][b, j] == 6
                assert o["finished"][b, j] and o["lengths"][b, j] == 0


def test_ties_go_to_the_lower_beam_the_larger_logit_the_lower_token():
    z = np.array([[[1.0, 2.0, 2.0], [1.0, 2.0, 2.0]]])
    o = O.select(z, np.zeros((1, 2)), 6)
    assert o["parents"].tolist() == [[0, 0, 1, 1, 0, 1]] and o["tokens"].tolist() == [[1, 2, 1, 2, 0, 0]]


def test_reorder_by_hand():
    s = np.arange(12).reshape(1, 4, 3)
    assert O.reorder(s, [[2, 2, -1, 0]]).tolist() == [[[6, 7, 8], [6, 7, 8], [6, 7, 8], [0, 1, 2]]]
    assert O.reorder(s, [[3, 9]], np.zeros((1, 2, 3))).tolist() == [[[9, 10, 11], [0, 0, 0]]]

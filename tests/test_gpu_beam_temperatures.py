"""aal_beam_select over the whole range of temperatures, 1e-37 to the largest fp32
number, against the fp64 oracle: choices are exact, scores and ranks to the tolerance
of test_gpu_beam.py.

log2(e) / T is held in two fp32 pieces. From T = 2^126 on they are multiples of 2^-149, so that what
they leave out is 2^-149 at most, which a logit of up to 2^128 makes 2^-21 of an exponent of two: 2^-21.5 of a
sum, within the 2^-20 there."""
import math

import pytest
import torch

from test_gpu_beam import A, BF16, F32, check  # noqa: F401

pytestmark = pytest.mark.gpu

LARGEST = torch.finfo(F32).max


def make(B, W, V, dtype, T, seed, masked):
    """Logits that are some units of T, or as many as the type holds; with masked, half of them are -inf and so is
    one whole row."""
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn(B, W, V, generator=g).double() * 2 * T).clamp(-torch.finfo(dtype).max, torch.finfo(dtype).max).to(dtype)
    if masked:
        z[torch.rand(B, W, V, generator=g) < 0.5] = -math.inf
        z[0, 1] = -math.inf
    return z, -torch.rand(B, W, generator=g).mul(2).cumsum(1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("T", [1e-37, 1e-20, 1e20, 1.2e36, 5e37, 8.5e37, 1e38, 2e38, 3e38, LARGEST])
def test_any_temperature(A, T, dtype, masked):  # noqa: F811
    """Rows of one part and of several, whose ends lie inside a vector."""
    T = torch.tensor(T).item()  # as the call takes it
    for V, n in ((5, 3), (1003, 4), (20_011, 16)):
        check(A, *make(2, 3, V, dtype, T, V, masked), n, T)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1e38, 3e38])
def test_logits_far_below_the_temperature(A, T, dtype):  # noqa: F811
    """Every allowed token is as likely as another: ties by beam, logit and token."""
    T = torch.tensor(T).item()
    for masked in (False, True):
        z, s = make(2, 3, 1003, dtype, 1.0, 4, masked)
        check(A, z, s, 7, T)

"""aal_topk_loss_fwd_bwd at the upper bound of every size of the resident schedule's workgroups
(waves that hold a row x 16-byte vectors a thread), for whole and ragged rows, every pair of element
types that it takes, and weights with and without a wait for other rows.

Tolerances against the oracle are those of test_gpu_topk_loss.py, which compares; between copies of a
window that different workgroups take, sums run in one order where rows are whole vectors (equal bits),
and at another phase of the vectors where they are ragged: the same tolerances for those, as bounds on
both sides, so twice 6 REL of the gradient's parts, of which no entry has more than four of at most q + p,
and 2^-7 of the bf16 value."""
import pytest
import torch

import test_gpu_topk_loss as loss

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
A = loss.A

SIZES = [(1, 9), (2, 9), (3, 12), (7, 9), (7, 14), (7, 19), (15, 14), (15, 17), (15, 20)]
LENGTHS = [(f"{wk}x{nv}{'' if whole else ' ragged'}", wk * 64 * nv, whole) for wk, nv in SIZES for whole in (True, False)]
TYPES = {"bf16": (BF16, BF16), "bf16-fp32": (BF16, F32), "fp32": (F32, F32)}


def lengths():
    for name, vectors, whole in LENGTHS:
        for types, (dtype, grad) in TYPES.items():
            e = 8 if dtype == BF16 else 4
            # a ragged row may start and end inside a vector, which counts as two more
            yield pytest.param(vectors * e if whole else (vectors - 2) * e + 3, dtype, grad, id=f"{name}-{types}")
    for V in (31999, 32000, 32001, 50257):
        yield pytest.param(V, BF16, BF16, id=f"{V}-bf16")


@pytest.mark.parametrize("weights,layout", [("all", loss.WIN), ("all", loss.SEQ), ("kl", loss.SEQ)],
                         ids=["windows", "sequences", "no wait"])
@pytest.mark.parametrize("V,dtype,grad", lengths())
def test_every_size_at_its_bound(A, V, dtype, grad, weights, layout):
    S, K, k = 4, (4 if layout == loss.WIN else 3), 6
    zd, top, ids, rest = loss.make(1, S, V, k, dtype, V)
    loss.check(A, zd, top, ids, rest, K, loss.WEIGHTS[weights], layout, grad_dtype=grad)
    # more rows than run at once: every workgroup takes several, their loads under the stores before
    n = 700 if V < 40000 else 300
    many = [t.repeat(n, *([1] * (t.dim() - 1))) for t in (zd, top, ids, rest)]
    got = A.aal_topk_loss_fwd_bwd(many[0], many[1], many[2], K, rest=many[3], weights=loss.WEIGHTS[weights], layout=layout,
                                  grad_dtype=grad, grad_scale=torch.tensor([float(n)], device="cuda"))
    one = A.aal_topk_loss_fwd_bwd(zd, top, ids, K, rest=rest, weights=loss.WEIGHTS[weights], layout=layout, grad_dtype=grad)
    whole = V % (8 if dtype == BF16 else 4) == 0
    accept = got["accept_tv"].view(n, S)
    torch.testing.assert_close(accept, one["accept_tv"].view(1, S).expand(n, S), rtol=4 * loss.REL, atol=4 * loss.REL)
    if whole:
        assert torch.equal(accept, accept[:1].expand(n, S))
        assert torch.equal(got["grad"], got["grad"][:1].expand_as(got["grad"]))
    size = one["grad"].float().abs().amax()
    for b in range(0, n, 100):  # in parts: the comparison's own copies are large
        g, h = got["grad"][b:b + 100].float(), one["grad"].float()
        tol = (2.0 ** -7 if grad == BF16 else 0.0) * h.abs() + 48 * loss.REL * size
        assert ((g - h).abs() <= tol).all()

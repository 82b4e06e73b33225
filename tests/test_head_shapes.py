"""The shapes that aal_head_logits_bwd refuses, whichever gradients it is asked for: checked before
anything touches a GPU."""
import pytest
import torch

import paper_2609_24150_amd as A

V, D, ROWS = 300, 200, 5


def head(*names, block_rows=128):
    n = lambda r: r if block_rows == 1 else (r + 127) // 128  # noqa: E731
    full = {"q": torch.zeros(V, D, dtype=torch.uint8).view(torch.float8_e4m3fn), "scale": torch.ones(n(V), 2),
            "qt": torch.zeros(D, V, dtype=torch.uint8).view(torch.float8_e4m3fn), "scale_t": torch.ones(n(D), 3)}
    return {k: full[k] for k in names or full}


@pytest.mark.parametrize("x_grad,weight_grad", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_logits_and_states_of_another_size(x_grad, weight_grad, block_rows):
    heads = [head(block_rows=block_rows), head("qt", "scale", "scale_t", block_rows=block_rows)]
    if not x_grad:
        heads += [head("q", "scale", block_rows=block_rows), head("scale", block_rows=block_rows)]
    for h in heads:
        sizes = [(V + 100, D), (V, D + 100)] if set(h) == {"scale"} else [(V - 1, D), (V + 1, D), (V, D - 1), (V, D + 1), (D, V)]
        for v, d in sizes:
            with pytest.raises(ValueError, match="do not fit a head"):
                A.aal_head_logits_bwd(torch.zeros(ROWS, v), torch.zeros(ROWS, d), h, x_grad=x_grad, weight_grad=weight_grad)
        # those of the head's go on to the next check, of where they are
        with pytest.raises(ValueError, match="on a device"):
            A.aal_head_logits_bwd(torch.zeros(ROWS, V), torch.zeros(ROWS, D), h, x_grad=x_grad, weight_grad=weight_grad)

"""aal_logits_process and aal_logits_process_bwd with histories as long as a length can be, where
an index of 32 bits with a sign would run over."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F32 = torch.float32


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_24150_amd as lib
    return lib


def test_histories_of_nearly_2_31_tokens(A):
    n, V = 2 ** 31 - 1, 16384
    tokens = torch.full((n + 9,), -1, dtype=torch.int32, device="cuda")  # outside the vocabulary: counted nowhere
    tokens[9], tokens[n + 8] = 5, 3  # the first and the last of the history
    z = torch.arange(1, V + 1, dtype=F32, device="cuda").view(1, V)  # sums, halves and differences are exact
    rules = dict(tokens=tokens, hist_start=torch.tensor([9], device="cuda"),
                 hist_len=torch.tensor([n], dtype=torch.int32, device="cuda"), repetition=torch.tensor([2.0], device="cuda"),
                 frequency=torch.tensor([0.25], device="cuda"), presence=torch.tensor([0.5], device="cuda"))
    for prompt in (None, n - 1, 1):
        if prompt is not None:
            rules["prompt_len"] = torch.tensor([prompt], dtype=torch.int32, device="cuda")
        want = z.clone()
        want[0, 5], want[0, 3] = z[0, 5] / 2, z[0, 3] / 2 - 0.75
        if prompt is None:
            want[0, 5] -= 0.75
        assert torch.equal(A.aal_logits_process(z, **rules), want)
        up = torch.ones_like(z)
        up[0, 5] = up[0, 3] = 0.5
        assert torch.equal(A.aal_logits_process_bwd(torch.ones_like(z), z, **rules), up)

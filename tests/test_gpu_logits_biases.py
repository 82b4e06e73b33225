"""aal_logits_process and aal_logits_process_bwd at the lengths of bias lists where their handling
changes (128 and 256 threads' worth of a round, 256 entries of the hash table) and far beyond, with
ids that occur again, against the fp64 oracle with the tolerances of test_gpu_logits.py."""
import pytest
import torch

import test_gpu_logits as logits

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
A = logits.A


def biases(counts, V, seed, distinct=False):
    """Bias lists of these lengths; ids from half as many values, so that most occur again, a
    twentieth of them outside the vocabulary."""
    g = torch.Generator().manual_seed(seed)
    n = torch.tensor(counts)
    ids = []
    for c in counts:
        if distinct:
            ids.append(torch.randperm(V, generator=g)[:c])
            continue
        some = torch.randint(0, V, (max(1, c // 2),), generator=g)
        i = some[torch.randint(0, len(some), (c,), generator=g)]
        i[torch.rand(c, generator=g) < 0.05] = -1
        i[torch.rand(c, generator=g) < 0.05] = V
        ids.append(i)
    return {"bias_offsets": torch.cat([n.new_zeros(1), n.cumsum(0)]), "bias_ids": torch.cat(ids).int(),
            "bias_values": torch.randn(int(n.sum()), generator=g) * 5}


def rules(counts, V, seed, **kw):
    r = logits.make_rules(len(counts), V, seed, hist=60, bias=0, masks=3)
    r.update(biases(counts, V, seed, **kw))
    return r


COUNTS = [0, 1, 127, 128, 129, 255, 256, 257, 500, 2000]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [1000, 1003, 4096, 5001, 9003, 33001, 128256])
def test_lists_of_every_length(A, V, dtype):
    counts = COUNTS + [3, 256, 0, 400]
    logits.check(A, logits.logits(len(counts), V, dtype, V), rules(counts, V, V), inplace=True)
    # alone, so that short calls and their grids come up too
    for c in (256, 257):
        logits.check(A, logits.logits(1, V, dtype, c), rules([c], V, c))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [1003, 20001])
def test_the_last_of_equal_ids_counts(A, V, dtype):
    # one id throughout, then two in turn, at lengths over one and over several rounds of a workgroup
    for c in (2, 130, 256, 257, 1500):
        r = rules([c] * 3, V, c)
        ids = torch.full((3, c), 7)
        ids[1, ::2] = V - 1
        ids[2, : c // 2] = torch.arange(c // 2) % V
        r["bias_ids"] = ids.view(-1).int()
        logits.check(A, logits.logits(3, V, dtype, c), r)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
def test_the_hash_table_at_its_fullest(A, dtype):
    # 256 different ids of one slice: the table half full; ids that share a place in it
    V = 4096
    r = rules([256] * 4, V, 1, distinct=True)
    place = (torch.arange(V) * 2654435761 % 2 ** 32 >> 16) % 512
    same = torch.argsort(place, stable=True)[:256]
    r["bias_ids"][:256] = same.int()
    r["bias_ids"][256:512] = torch.arange(256).int()
    logits.check(A, logits.logits(4, V, dtype, 2), r, inplace=True)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [3001, 40000])
def test_long_lists_with_long_histories(A, V, dtype):
    # counters of 32 bits for both reasons, in one call with rows that need neither
    counts = [300, 0, 300, 2, 1000]
    r = rules(counts, V, 5)
    n = 33000
    words = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(6))
    words[::3] = 17
    r.update(tokens=words.int(), hist_start=torch.tensor([0, 0, 5, 100, 0]),
             hist_len=torch.tensor([n, n, 40, 70, n]).int(), prompt_len=torch.tensor([0, 1, 20, 0, 300]).int())
    logits.check(A, logits.logits(len(counts), V, dtype, 3), r, inplace=True)


@pytest.mark.parametrize("z_dtype,g_dtype", [(BF16, F32), (F32, BF16)])
def test_gradient_types(A, z_dtype, g_dtype):
    counts = [300, 10, 256, 700]
    logits.check(A, logits.logits(len(counts), 5003, z_dtype), rules(counts, 5003, 3), g_dtype=g_dtype)

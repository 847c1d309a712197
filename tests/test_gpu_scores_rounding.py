"""Softmax weights summed per cached token where scores are large: a row gives out what its own sum was made of, whichever kernel made that sum."""
import pytest
import torch

pytestmark = pytest.mark.gpu

cg = pytest.importorskip("paper_2512_17970_amd")
from attention_util import counters_are_clear, starts, workspace  # noqa: E402
from gpu_util import stream  # noqa: E402
from test_gpu_attention_scores import FP16, FP8, INT4, INT8, make, queries, sequence  # noqa: E402

TYPES = [(FP16, 1), (INT8, 16), (FP8, 1), (INT4, 32)]
# The largest score of a call, times log2(e), which fp32 rounds by up to 2^-12, 2^-8, 2^-5, 2^-4 and 32.
LARGEST = [7000.0, 1e5, 2.0 ** 20 - 1, 2.0 ** 20 + 40, 1e9]


def given_out(c, q, new, largest, single):
    """Per sequence the sums over its tokens [heads] in 64 bits, of a call whose largest score is `largest`."""
    r, at, most = q.shape[1] // c.heads, 0, 0.0
    for i, n in enumerate(new):
        k, _ = sequence(c, i, 0, c.lens[i])
        for h in range(c.heads):
            most = max(most, float((k[:, h] @ q[at:at + n, h * r:(h + 1) * r].double().flatten(0, 1).T).abs().max()))
        at += n
    desc = cg.AttnDesc.make(q.shape[1], c.heads, c.dim, num_seqs=len(new), total_q=len(q), max_kv=max(c.lens), scale=largest / (most * 1.4426950408889634))
    s = c.struct()
    scores = torch.zeros(c.pages, c.heads, c.page, device="cuda")
    if single:
        ws, n = workspace(cg.codegemm_attn_decode_scores_workspace_bytes(s, desc))
        cg.codegemm_attn_decode_scores(s, desc, q, torch.empty_like(q), None, None, scores, ws, n, stream())
    else:
        ws, n = workspace(cg.codegemm_attn_scores_workspace_bytes(s, desc))
        cg.codegemm_attn_scores(s, desc, q, starts(new), None, None, scores, ws, n, stream())
    assert counters_are_clear()
    return [sum(scores[c.page_of(i, t), :, t % c.page].double() for t in range(c.lens[i])) for i in range(len(new))]


def off(got, rows, n):
    """How far sums over n tokens of `rows` weights are from `rows`, in units of what they may be off by.  A weight and a row's sum of them are made of the same scores, so what these
    are rounded by does not count.  What does: an exponential (2^-23), its argument's rounding, which takes at most 2^-24 of the row (w |log2 w| ln 2 < 0.54), factors that join parts (2^-22),
    the sum's roundings (fewer than n + 32 of 2^-24), 1 / sum and the product with it (2^-23), and as many roundings as there are rows in a token's sum."""
    return float((got - rows).abs().max() / (rows * (n + 64 + rows) * 2.0 ** -24))


@pytest.mark.parametrize("dtype,block", TYPES)
@pytest.mark.parametrize("largest", LARGEST)
def test_few_queries(dtype, block, largest):
    """Up to 16 rows of a key head in a call: their sums by one kernel, their weights by that for few rows; sequences of one token, whose weight is 1, and longer ones."""
    for lens, new, heads, group, dim in (([1, 1, 37], [1, 1, 1], 2, 4, 64), ([1, 290], [1, 1], 1, 8, 128), ([140], [3], 1, 5, 128), ([1], [1], 1, 16, 256)):
        c = make(lens, dtype, heads=heads, dim=dim, block=block, page=64, seed=len(lens))
        got = given_out(c, queries(sum(new), heads * group, dim, seed=int(largest) % 1000), new, largest, False)
        for x, n, rows in zip(got, lens, new):
            assert off(x, rows * group, n) <= 1, (lens, n, off(x, rows * group, n))


@pytest.mark.parametrize("dtype,block", TYPES)
@pytest.mark.parametrize("largest", LARGEST)
def test_single_tokens_of_many_query_heads(dtype, block, largest):
    """More than 16 query heads to a key head: their sums by the attention, their weights by the kernel for many rows."""
    for lens, heads, group, dim in (([1, 37, 270], 1, 20, 64), ([1, 290], 2, 17, 128), ([5, 1], 1, 40, 128)):
        c = make(lens, dtype, heads=heads, dim=dim, block=block, page=64, seed=len(lens))
        got = given_out(c, queries(len(lens), heads * group, dim, seed=int(largest) % 1000), [1] * len(lens), largest, True)
        for x, n in zip(got, lens):
            assert off(x, group, n) <= 1, (lens, n, off(x, group, n))


@pytest.mark.parametrize("dtype,block", TYPES)
@pytest.mark.parametrize("largest", LARGEST)
def test_the_other_pairs(dtype, block, largest):
    """Many rows after their own sums, few after the attention's."""
    for lens, new, heads, group, dim in (([1, 37, 270], [1, 20, 8], 1, 4, 64), ([290], [40], 2, 3, 128)):
        c = make(lens, dtype, heads=heads, dim=dim, block=block, page=64, seed=len(lens))
        got = given_out(c, queries(sum(new), heads * group, dim, seed=int(largest) % 1000), new, largest, False)
        for x, n, rows in zip(got, lens, new):
            assert off(x, rows * group, n) <= 1, (lens, n, off(x, rows * group, n))
        q = queries(len(lens), heads * group, dim, seed=3)
        for x, n in zip(given_out(c, q, [1] * len(lens), largest, True), lens):
            assert off(x, group, n) <= 1, (lens, n, off(x, group, n))

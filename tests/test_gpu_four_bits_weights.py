"""Softmax weights far below the largest over a cache in 4 bits: one key that takes most of the weight and has values of zero, and thousands of equal keys whose small
weights make the whole result; scores so large that one key has all the weight.  Against the definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

cg = pytest.importorskip("paper_2512_17970_amd")
from four_bits_util import Cache4, pack  # noqa: E402
from test_gpu_attention_weights import bound, column, sink_query  # noqa: E402
from test_gpu_four_bits import decode  # noqa: E402

N = 50000


def codes_of(x):
    """[dim] of codes -> words [dim / 8]"""
    return pack(x.view(-1, 8)).cuda()


def value_words(code):
    """Values' words of 16 equal tokens: [dim][2]"""
    return pack(code[:, None, None].expand(-1, 2, 8)).cuda()


def sink_cache(n, at, dim, page=64, heads=1, seqs=1):
    """n + 1 tokens, all keys zero but that of token `at`, which has 4 in dimension 0 and values of zero; the others' values are those of `column`, which are 1 + code / 8."""
    c = Cache4([n + 1] * seqs, heads=heads, dim=dim, page=page, block=32, filled=[0] * seqs, quick=True)
    c.k.zero_()
    c.k_scales[..., 0], c.k_scales[..., 1] = 0.5, -8.0                   # (0 + 16) / 2 - 8 = 0
    c.v.copy_(value_words(torch.arange(dim) % 8).expand_as(c.v))
    c.v_scales[..., 0, :], c.v_scales[..., 1, :] = 0.125, -1.0           # (code + 16) / 8 - 1
    key = torch.zeros(dim, dtype=torch.long)
    key[0] = 8                                                          # 24 / 2 - 8
    for i in range(seqs):
        p, s = c.page_of(i, at), at % page
        c.k[p, :, s] = codes_of(key)
        c.v_scales[p, :, s // 16, :, :, s % 16] = 0.0
        for t in range(n + 1, -(-(n + 1) // page) * page):               # behind the last token
            p, s = c.page_of(i, t), t % page
            c.v_scales[p, :, s // 16, :, :, s % 16] = float("nan")
            c.k_scales[p, :, s] = float("nan")
    return c


def close(got, gap, n, dim):
    w = n * math.exp(-gap)
    want = w / (1 + w) * column(dim)
    error = float(((got.double() - want).abs() / want).max())
    assert error <= bound(n), f"{gap} nats: {error:.1e}, {error / bound(n):.2f} times the bound"


@pytest.mark.parametrize("dim,page", [(128, 64), (64, 16), (96, 32), (256, 256)])
@pytest.mark.parametrize("at", [0, 20011, N])
def test_small_weights_behind_a_sink(dim, page, at):
    c, q = sink_cache(N, at, dim, page), sink_query(8, dim)
    for gap in (5.0, 10.0, 12.5, 14.0, 15.0, 16.0, 17.0, 18.0):
        close(decode(c, q, scale=gap / 32), gap, N, dim)


@pytest.mark.parametrize("dim", [64, 128])
def test_small_weights_behind_a_sink_in_one_workgroup(dim):
    n = 6000
    c, q = sink_cache(n, 0, dim, heads=60, seqs=5), sink_query(60, dim, 5)
    for gap in (5.0, 10.0, 12.5, 14.0, 15.0, 16.0, 17.0):
        close(decode(c, q, scale=gap / 32), gap, n, dim)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("step", [0.5, 3.0, 5.0, 6.0, 11.0, 100.0])
def test_maxima_that_grow_from_key_to_key(dim, step):
    """Scores that rise by `step` (base 2) every 100 tokens, and fall again: the weights behind each rise are small beside what comes."""
    n = 3000
    c = Cache4([n], heads=1, dim=dim, page=64, block=32, filled=[0], quick=True)
    c.k.zero_()
    c.v.copy_(value_words(torch.arange(dim) % 8).expand_as(c.v))
    c.v_scales[..., 0, :], c.v_scales[..., 1, :] = 0.125, -1.0
    c.k_scales.zero_()
    key = torch.zeros(n, dtype=torch.float64)
    for t in range(n):
        level = t // 100 if t < 2000 else 39 - t // 100                  # up to 19, then down
        p, s = c.page_of(0, t), t % 64
        c.k_scales[p, :, s, :, 1] = float(level)                          # all codes 0, scale 0: the key is its offset
        key[t] = level
        c.v_scales[p, :, s // 16, :, 0, s % 16] = 0.125 * (1 + level % 3)
        c.v_scales[p, :, s // 16, :, 1, s % 16] = -1.0 * (1 + level % 3)  # (1 + level % 3) times the column
    q = torch.zeros(1, 8, dim, dtype=torch.float16, device="cuda")
    q[..., 0] = 1.0
    p = torch.softmax(key * step * math.log(2.0), 0)
    want = float((p * (1 + key % 3)).sum()) * column(dim)
    got = decode(c, q, scale=step * math.log(2.0)).double()
    # weights and result rounded to 11 bits; a score of up to 1900 in base 2 is off by its own rounding and the scale's, 2^-23 of it
    assert float(((got - want).abs() / want).max()) <= 2.0 ** -10 + 2 * 19 * step * 2.0 ** -23 + 3 * n / 32 * 2.0 ** -24


@pytest.mark.parametrize("size", [100.0, 3000.0, 60000.0])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("dim", [64, 128])
def test_large_scores(size, sign, dim):
    """Keys and queries of up to 60000: one key has all the weight, whatever the scores' sign."""
    n = 500
    c = Cache4([n], heads=1, dim=dim, page=32, block=32, filled=[0], quick=True)
    c.k.zero_()
    c.k_scales[..., 0], c.k_scales[..., 1] = 0.0, sign * size
    best = 333
    for t in range(n):
        p, s = c.page_of(0, t), t % 32
        c.v_scales[p, :, s // 16, :, 0, s % 16], c.v_scales[p, :, s // 16, :, 1, s % 16] = 0.0, t / 4
        if (t == best) == (sign < 0):
            c.k_scales[p, :, s, :, 1] = sign * size / 2                  # the least of the negative ones, all but the largest of the positive
    q = torch.full((1, 4, dim), size, dtype=torch.float16, device="cuda")
    got = decode(c, q, scale=1.0)
    assert bool((got.double() == best / 4).all())

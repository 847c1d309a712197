"""Softmax weights far below the largest: one key that takes most of the weight and has values of zero, and tens of thousands of equal keys whose small
weights make the whole result; scores beyond the range in which 32 bits hold their fractions.  Against the definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

cg = pytest.importorskip("paper_2512_17970_amd")
from attention_util import Cache, decode, prompt  # noqa: E402

FP16, INT8, FP8 = cg.binding.KV_FP16, cg.binding.KV_INT8, cg.binding.KV_FP8
N = 50000
EMPTY = [0] * 4100          # sequences without tokens: as many tiles as keep the keys of one from being shared


def bound(n):
    """Relative error of a result that n equal weights make: a weight's rounding to fp16 (2^-11, all of them the same way) and the result's (2^-11); a score of
    up to 30 in base 2 is off by 30 2^-23 ln 2 at most, its exponential by two units of 2^-23; sums in 32 bits add n / 32 products of 32 keys to one another in
    turn, and twice as many times a handful of weights to the sum of all, of which one may be far larger: 3 n / 32 2^-24 (with the former, 2^-11 at least)."""
    return 2.0 ** -10 + max(2.0 ** -11, 3 * n / 32 * 2.0 ** -24)


def column(dim):
    """Values of the equal keys, one for each dimension; exact in fp16, and times 64 in int8; of 3 bits of mantissa."""
    return (torch.arange(dim) % 8 + 8).double().cuda() / 8


def close(got, gap, n, dim):
    """got [..][dim]; n equal keys `gap` nats under the one whose values are zero."""
    w = n * math.exp(-gap)
    want = w / (1 + w) * column(dim)
    error = float(((got.double() - want).abs() / want).max())
    assert error <= bound(n), f"{gap} nats: {error:.1e}, {error / bound(n):.2f} times the bound"


def sink_cache(n, at, dim, dtype, block, heads=1, seqs=1):
    """n + 1 tokens, all keys zero but that of token `at`, which has 4 in dimension 0 and values of zero."""
    c = Cache([n + 1] * seqs, heads=heads, dim=dim, page=64, dtype=dtype, block=block, filled=[0] * seqs)
    one, v = {FP16: (1.0, column(dim).half()), INT8: (64.0, (column(dim) * 64).to(torch.int8).view(torch.uint8)),
              FP8: (1.0, column(dim).to(torch.float8_e4m3fn).view(torch.uint8))}[dtype]
    c.k.zero_()
    c.v.copy_(v[:, None].expand_as(c.v))
    key = torch.zeros(1, dim, device="cuda")
    key[0, 0] = 4.0
    if dtype == FP16:
        key = key.half()
    else:
        c.k_scales.fill_(1 / 16 if dtype == INT8 else 1.0)
        c.v_scales.fill_(1 / one)
        key = (key * 16).to(torch.int8).view(torch.uint8) if dtype == INT8 else key.to(torch.float8_e4m3fn).view(torch.uint8)
    for i in range(seqs):
        c.place(c.k, i, at, False).copy_(key.expand(heads, dim))
        c.place(c.v, i, at, True).zero_()
        for t in range(n + 1, -(-(n + 1) // 64) * 64):                   # behind the last token
            c.place(c.v, i, t, True).fill_(float("nan") if dtype == FP16 else 0x7F)
    return c


def sink_query(heads, dim, seqs=1):
    q = torch.zeros(seqs, heads, dim, dtype=torch.float16, device="cuda")
    q[:, :, 0] = 8.0
    return q


@pytest.mark.parametrize("dtype,block,dim", [(FP16, 1, 64), (FP16, 1, 256), (INT8, 16, 128), (INT8, 1, 64), (INT8, 4, 80), (FP8, 64, 128), (FP8, 1, 64)])
@pytest.mark.parametrize("at", [0, 20011, N])
def test_decode_small_weights_behind_a_sink(dtype, block, dim, at):
    c, q = sink_cache(N, at, dim, dtype, block), sink_query(8, dim)
    for gap in (5.0, 10.0, 12.5, 14.0, 15.0, 16.0, 17.0, 18.0):
        close(decode(c, q, scale=gap / 32), gap, N, dim)


@pytest.mark.parametrize("dtype,block,dim", [(FP16, 1, 64), (FP16, 1, 128), (INT8, 16, 128), (INT8, 16, 64), (INT8, 4, 80), (FP8, 64, 128), (FP8, 16, 256)])
def test_decode_small_weights_behind_a_sink_in_one_workgroup(dtype, block, dim):
    """More items than compute units: none is cut, and a wavefront has a quarter or half of a sequence's keys."""
    n = 6000
    c, q = sink_cache(n, 0, dim, dtype, block, heads=60, seqs=5), sink_query(60, dim, 5)
    for gap in (5.0, 10.0, 12.5, 14.0, 15.0, 16.0, 17.0):
        close(decode(c, q, scale=gap / 32), gap, n, dim)


def sink_prompt(n, at, dim):
    k, v = torch.zeros(n + 1, 1, dim, dtype=torch.float16, device="cuda"), column(dim).half().expand(n + 1, 1, dim).contiguous()
    k[at, 0, 0] = 4.0
    v[at] = 0
    return k, v


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("at", [0, 20011, N])
@pytest.mark.parametrize("shared", [True, False])
def test_prompt_small_weights_behind_a_sink(dim, at, shared):
    """Keys of a tile of queries shared by several workgroups, and not."""
    k, v = sink_prompt(N, at, dim)
    q = sink_query(4, dim).expand(40, 4, dim).contiguous()
    beside = [] if shared else EMPTY
    for gap in (5.0, 10.0, 12.5, 14.0, 15.0, 16.0, 17.0, 18.0):
        close(prompt(q, k, v, [40] + beside, [N + 1] + beside, scale=gap / 32, causal=False), gap, N, dim)


@pytest.mark.parametrize("dim", [64, 128])
def test_prompt_small_weights_in_masked_tiles(dim):
    """The sink is the last key that all queries see; the equal keys in front of it are seen in part by the window."""
    n, gap = 3000, 14.0
    k, v = sink_prompt(n, n, dim)
    q = sink_query(2, dim).expand(64, 2, dim).contiguous()
    k, v = torch.cat([k, torch.zeros_like(k[:63])]), torch.cat([v, v[:63]])
    got = prompt(q, k, v, [64], [n + 64], scale=gap / 32, window=2000)
    for i in range(64):                                                  # query i sees the 2000 keys up to n + i, the sink among them
        close(got[i], gap, 1999, dim)


@pytest.mark.parametrize("below", [20, 24, 27, 28, 30])
def test_decode_weights_that_are_powers_of_two(below):
    """A million keys a power of two below the sink."""
    n, dim, ln2 = 1 << 20, 64, math.log(2.0)
    for at in (0, n):
        close(decode(sink_cache(n, at, dim, FP16, 1), sink_query(2, dim), scale=below * ln2 / 32), below * ln2, n, dim)


@pytest.mark.parametrize("below", [20, 24, 27, 28, 30])
def test_prompt_weights_that_are_powers_of_two(below):
    n, dim, ln2 = 1 << 20, 64, math.log(2.0)
    for at in (0, n):
        k, v = sink_prompt(n, at, dim)
        for beside in ([], EMPTY):
            close(prompt(sink_query(2, dim), k, v, [1] + beside, [n + 1] + beside, scale=below * ln2 / 32, causal=False), below * ln2, n, dim)


@pytest.mark.parametrize("size", [100.0, 1000.0, 8000.0, 60000.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_scores_beyond_all_fractions(size, sign, dim):
    """Keys and queries up to the largest of fp16, scores up to 10^12, of which 32 bits hold no fraction: the one key whose score is the largest by far has all
    the weight."""
    n, heads, best = 700, 4, 333
    g = torch.Generator().manual_seed(int(size) + dim)
    signs = torch.where(torch.rand(dim, generator=g) < 0.5, -1.0, 1.0)
    amount = torch.rand(n, generator=g) * 0.5                            # of positive scores; of negative ones 0.5 to 1, and the least for the largest
    amount[best] = 1.0
    if sign < 0:
        amount = -(amount + 0.5)
        amount[best] = -0.25
    jitter = 1 + torch.rand(heads, generator=g) * 2.0 ** -4              # products with many places
    q = (signs * jitter[None, :, None] * 0.9 * size).half().cuda()
    k = (signs * amount[:, None, None] * size).half().cuda()
    v = torch.randn(n, 1, dim, generator=g).half().cuda()
    scale = dim ** -0.5
    first, second = ((q[0].double() @ k[:, 0].double().t()) * scale).topk(2, dim=1).values.unbind(1)
    assert bool((first - second > 0.2 * torch.maximum(first.abs(), second.abs())).all()) and float((first - second).min()) > 1000
    want = v[best, 0]
    for beside in ([], EMPTY):
        for rows in (1, 60):
            got = prompt(q.expand(rows, heads, dim).contiguous(), k, v, [rows] + beside, [n] + beside, scale=scale, causal=False)
            assert torch.equal(got, want.expand_as(got)), f"prompt of {rows}"
    c = Cache([n], heads=1, dim=dim, page=64, dtype=FP16, filled=[0])
    for t in range(n):
        c.place(c.k, 0, t, False).copy_(k[t])
        c.place(c.v, 0, t, True).copy_(v[t])
    got = decode(c, q, scale=scale)
    assert torch.equal(got, want.expand_as(got)), "decode"


@pytest.mark.parametrize("scale", [3.4e38, 1e30, 1e20, -1e30, -3.4e38])
@pytest.mark.parametrize("dtype,block,dim", [(FP16, 1, 64), (INT8, 16, 128), (FP8, 1, 256)])
def test_any_finite_scale(scale, dtype, block, dim):
    """The largest score (of a negative scale, the smallest) has all the weight."""
    n, heads = 300, 4
    c = Cache([n], heads=1, dim=dim, page=64, dtype=dtype, block=block, seed=5)
    k, v = (torch.stack([c.read(0, t, values) for t in range(n)]) for values in (False, True))
    q = (torch.randn(1, heads, dim, generator=torch.Generator().manual_seed(3)) * 2).half().cuda()
    scores = q[0].double() @ k[:, 0].t() * math.copysign(1, scale)
    first, second = scores.topk(2, dim=1).values.unbind(1)
    assert float((first - second).min()) > 1e-3 * float(scores.abs().max())
    want = v[scores.argmax(dim=1), 0]
    got = decode(c, q, scale=scale)[0].double()
    assert bool(((got - want).abs() <= 2.0 ** -10 * want.abs() + 2.0 ** -25).all()), "decode"      # the rounding of a weight with its scale, and the result's
    if dtype == FP16:
        for beside in ([], EMPTY):
            got = prompt(q, k.half(), v.half(), [1] + beside, [n] + beside, scale=scale, causal=False)
            assert torch.equal(got[0].double(), want), "prompt"


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 300])
def test_rows_of_all_sizes_beside_each_other(dim, window):
    """Queries whose scores are of sizes from 0.01 to some millions lie in one tile, and each is right for itself.  With p the weights and o the result in 64 bits,
    weights that are off by a factor of up to 1 + d each change it by 2 d / (1 - d) sum p |v - o| at most; d: a score's error, (D + 4) 2^-24 of its products'
    sizes, a weight's rounding and its exponential's.  Sums in 32 bits add (n + 64) 2^-24 sum p |v|, weights under 2^-34 of the largest n 2^-33 max |v|."""
    n, heads = 900, 2
    g = torch.Generator().manual_seed(dim + window)
    size = 10.0 ** (torch.arange(n * heads) % 9 - 4).view(n, heads, 1)
    k, v = ((torch.randn(n, 1, dim, generator=g) * s).half().cuda() for s in (100.0, 1.0))
    q = (torch.randn(n, heads, dim, generator=g) * size).half().cuda()
    scale = dim ** -0.5
    got = [prompt(q, k, v, [n] + beside, [n] + beside, scale=scale, window=window).double() for beside in ([], EMPTY)]
    key, at = torch.arange(n, device="cuda"), torch.arange(n, device="cuda")[:, None]
    seen, values = (key <= at) & ((key > at - window) if window else True), v[:, 0].double()
    for h in range(heads):
        s = (q[:, h].double() @ k[:, 0].double().t() * scale).masked_fill(~seen, -math.inf)
        error = (dim + 4) * 2.0 ** -24 * (scale * q[:, h].double().abs() @ k[:, 0].double().abs().t()).masked_fill(~seen, 0).amax(1)
        p = torch.softmax(s, dim=1)
        want = p @ values
        spread = torch.cat([(p[i:i + 50, :, None] * (values[None] - want[i:i + 50, None]).abs()).sum(1) for i in range(0, n, 50)])
        known = error < 0.1                                                # .. where 32 bits say something of a score's fraction
        d = (torch.expm1(error) + 2.0 ** -11 + 2.0 ** -16)[:, None]
        bound_ = 2 * d / (1 - d) * spread + (n + 64) * 2.0 ** -24 * (p @ values.abs()) + n * 2.0 ** -33 * values.abs().max() + 2.0 ** -11 * want.abs() + 2.0 ** -25
        first, second = s[1:].topk(2, dim=1).values.unbind(1)
        alone = torch.cat([torch.ones(1, dtype=torch.bool, device="cuda"), first - second > 40 + 4 * error[1:]])
        assert int(known.sum()) > n / 2 and int((alone & ~known).sum()) > n / 4
        for out in got:
            bad = (((out[:, h] - want).abs() > 1.01 * bound_) & known[:, None]).any(1)
            assert not bool(bad.any()), f"head {h}: rows {bad.nonzero()[:8, 0].tolist()}"
            assert torch.equal(out[alone, h], values[s.argmax(1)[alone]]), "rows of one key"

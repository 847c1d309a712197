"""codegemm_kv_evict where it takes its other ways: sequences that several workgroups select from, of several key heads, and moves of many places to a workgroup."""
import pytest
import torch

pytestmark = pytest.mark.gpu

cg = pytest.importorskip("paper_2512_17970_amd")
from attention_util import QMAX  # noqa: E402
from four_bits_util import Cache4, unpack  # noqa: E402
from test_gpu_eviction import FP16, FP8, INT4, INT8, evict, make  # noqa: E402


def kept(c, i, scores, budget, first, last):
    """Positions [heads][m] that sequence i keeps, by sorts: from the highest score down, NaN behind all, the lower position first."""
    n = max(0, c.lens[i])
    t = torch.arange(n)
    page = torch.where(t < c.max_pages * c.page, c.table[i, (t // c.page).clamp(max=c.max_pages - 1)].long(), -1)
    there = t[(page >= 0) & (page < c.pages)]
    if len(there) <= budget:
        return there.expand(c.heads, -1).cuda()
    always = (there < first) | (there >= n - last)
    others, out = there[~always], []
    for h in range(c.heads):
        s = scores[page[others].cuda(), h, (others % c.page).cuda()].cpu().double()
        nan = s.isnan()
        order = torch.sort(torch.where(nan, 0.0, -s), stable=True).indices
        order = order[torch.sort(nan[order].int(), stable=True).indices]
        out.append(torch.cat([there[always], others[order[:budget - int(always.sum())]]]).sort().values)
    return torch.stack(out).cuda()


def places(c, i, t):
    """pages and slots of positions t [heads][m] of sequence i, and the heads beside them"""
    return c.table.cuda()[i].long()[t // c.page], torch.arange(c.heads, device="cuda")[:, None], t % c.page


def rows(c, i, t, values):
    """codes or halves [heads][m][dim] of positions t"""
    p, h, s = places(c, i, t)
    if isinstance(c, Cache4):
        if not values:
            return unpack(c.k[p, h, s]).flatten(-2)
        return torch.gather(unpack(c.v[p, h, s // 16, :, s % 16 // 8]), -1, (s % 8)[..., None, None].expand(*s.shape, c.dim, 1))[..., 0]
    return c.v[p, h, s // 16, :, s % 16] if values else c.k[p, h, s]


def scales(c, i, t, values):
    p, h, s = places(c, i, t)
    if isinstance(c, Cache4):
        return c.v_scales[p, h, s // 16, :, :, s % 16] if values else c.k_scales[p, h, s]
    pool = c.v_scales if values else c.k_scales
    return None if pool is None else pool[p, h, s // c.block]


def bits(x):
    return x.contiguous().view(torch.uint8)


def run(c, scores, budget, first=0, last=0, max_kv=None):
    stay = [kept(c, i, scores, budget, first, last) for i in range(len(c.lens))]
    lens = [s.shape[1] for s in stay]
    to = make(lens, c.dtype, heads=c.heads, dim=c.dim, page=c.page, block=c.block, seed=99, filled=[0] * len(lens))
    old = [None if x is None else x.clone() for x in (to.k, to.k_scales, to.v, to.v_scales)]
    got, shift, new = evict(c, to, scores, budget, first, last, max_kv)
    assert got.tolist() == lens and shift.tolist() == [max(0, n) - m for n, m in zip(c.lens, lens)]
    expect = torch.full_like(new, -7.0)
    for i, src in enumerate(stay):
        m = src.shape[1]
        dst = torch.arange(m, device="cuda").expand(c.heads, m)
        a, b = places(c, i, src), places(to, i, dst)
        expect[b[0], b[1], b[2]] = scores[a[0], a[1], a[2]]
        for values in (False, True):
            x, y, s, z = rows(c, i, src, values), rows(to, i, dst, values), scales(c, i, src, values), scales(to, i, dst, values)
            if c.dtype in (FP16, INT4) or c.block == 1:
                assert torch.equal(bits(x), bits(y)) and (s is None or torch.equal(bits(s), bits(z))), (i, values)
                continue
            # a block has the largest scale of the tokens that come into it, and their codes in it
            pad = torch.nn.functional.pad(s, (0, -m % c.block))
            assert torch.equal(z, pad.unflatten(-1, (-1, c.block)).amax(-1).repeat_interleave(c.block, -1)[:, :m]), (i, values)
            same = (s == z)[..., None].expand(x.shape)
            assert torch.equal(x[same], y[same])
            want = c.value(x.contiguous()) * (s / z).double()[..., None]
            half = 0.5 if c.dtype == INT8 else want.abs() * 2.0 ** -4 + 2.0 ** -10          # half a step: of integers; of 3 bits of mantissa, and of the least numbers
            assert bool(((c.value(y.contiguous()) - want).abs() <= half + 2.0 ** -23 * QMAX[c.dtype]).all()), (i, values)       # (s / z and its product each rounded to 24 bits)
    assert torch.equal(expect.view(torch.int32), new.view(torch.int32))
    # nothing else was written
    for i, m in enumerate(lens):
        dst = torch.arange(m, device="cuda").expand(c.heads, m)
        p, h, s = places(to, i, dst)
        if isinstance(to, Cache4):
            for pool, now, nib in ((old[0], to.k, False), (old[2], to.v, True)):
                if not nib:
                    pool[p, h, s] = now[p, h, s]
                    continue
                # a word holds eight tokens; those that are none keep their codes
                live = torch.zeros(pool.shape[:3] + (16,), dtype=torch.bool, device="cuda")
                live[p, h, s // 16, s % 16] = True
                mask = (live.view(*live.shape[:3], 1, 2, 8).long() * torch.tensor([15 << (4 * (j // 2) + 16 * (j % 2)) for j in range(8)], device="cuda")).sum(-1)
                mask = torch.where(mask >= 1 << 31, mask - (1 << 32), mask).to(torch.int32)
                pool.copy_((pool & ~mask) | (now & mask))
            old[1][p, h, s] = to.k_scales[p, h, s]
            old[3][p, h, s // 16, :, :, s % 16] = to.v_scales[p, h, s // 16, :, :, s % 16]
            continue
        old[0][p, h, s] = to.k[p, h, s]
        old[2][p, h, s // 16, :, s % 16] = to.v[p, h, s // 16, :, s % 16]
        if old[1] is not None:
            old[1][p, h, s // c.block] = to.k_scales[p, h, s // c.block]
            old[3][p, h, s // c.block] = to.v_scales[p, h, s // c.block]
    for x, y in zip(old, (to.k, to.k_scales, to.v, to.v_scales)):
        assert x is None or torch.equal(bits(x), bits(y)), "a place that is no token's was written"


def some(c, kind, seed=1):
    g = torch.Generator().manual_seed(seed)
    shape = (c.pages, c.heads, c.page)
    x = torch.rand(shape, generator=g)
    if kind == "equal":
        x = torch.full(shape, 0.75)
    elif kind == "sums":                                      # of weights: a few have most, thousands the same
        x = (x ** 8 * 4096).round() / 4096
    elif kind == "close":                                     # they differ in the last bits only
        x = (torch.full(shape, 1.0).view(torch.int32) + torch.randint(0, 700, shape, generator=g).int()).view(torch.float32)
    elif kind == "odd":
        odd = torch.tensor([float("nan"), float("inf"), float("-inf"), -0.0, 0.0, -1.0, -2.5, 1e-40, -1e-40, 3e38, 1e-45, 0.5])
        x = odd[torch.randint(0, len(odd), shape, generator=g)]
    elif kind == "negative":
        x = -x
    elif kind == "few":                                       # a hundred have something, the rest nothing
        x = torch.where(x > 0.998, x, 0.0)
    return x.cuda()


@pytest.mark.parametrize("kind", ["equal", "sums", "close", "odd", "negative", "few"])
@pytest.mark.parametrize("budget,first,last", [(10000, 7, 50), (300, 100, 200), (25000, 0, 0), (1, 0, 0), (39999, 0, 39999), (1 << 30, 5, 5)])
def test_selected_from_by_several_workgroups(kind, budget, first, last):
    """Five workgroups to each of two key heads of 40000 tokens; budget = first + last leaves room for no others.  Shorter sequences beside it, of which some of the five have nothing."""
    c = Cache4([40000, 100, 0, 20011], heads=2, dim=32, page=64, seed=3)
    run(c, some(c, kind), budget, first, last)


@pytest.mark.parametrize("kind", ["equal", "sums", "odd"])
@pytest.mark.parametrize("budget,first,last", [(9000, 300, 300), (600, 300, 300), (1 << 30, 0, 0)])
def test_pages_that_are_not_there_where_workgroups_meet(kind, budget, first, last):
    """Parts of 8000 positions: pages of 256 across their ends, a whole part, the first and the last page."""
    c = Cache4([40000, 33000], heads=3, dim=32, page=256, seed=5)
    for j in (0, 31, 32, 62, *range(94, 125), 156):
        c.table[0, j] = -1 if j % 2 else c.pages + 7
    c.table[1, 128] = -3
    c.table_dev.copy_(c.table.cuda())
    run(c, some(c, kind), budget, first, last)


@pytest.mark.parametrize("max_kv", [16385, 1 << 30])
def test_lengths_that_the_host_does_not_know(max_kv):
    """Parts of more positions than LDS holds, and more parts than there are positions for."""
    c = Cache4([50000, 5], heads=1, dim=32, page=64, seed=6)
    run(c, some(c, "sums"), 20000, 4, 64, max_kv=max_kv)


@pytest.mark.parametrize("dtype,block", [(FP16, 1), (INT8, 1), (INT8, 4), (INT8, 64), (FP8, 2), (FP8, 16), (INT4, 32)])
@pytest.mark.parametrize("dim", [32, 64])
def test_many_places_to_a_workgroup(dtype, block, dim):
    """16 sequences of 16 key heads that keep 530 tokens: more than 4096 workgroups of 64 places, so these take 256."""
    lens = [601, 530, 0, 20, 1, 577, 256, 257] + [3] * 8
    c = make(lens, dtype, heads=16, dim=dim, block=block, page=64, seed=dim)
    run(c, some(c, "sums"), 530, 4, 40)

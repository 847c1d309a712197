"""codegemm_kv_evict against its definition: which tokens stay, where they go, what is moved and what is left as it was."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

cg = pytest.importorskip("paper_2512_17970_amd")
from attention_util import Cache, counters_are_clear, workspace  # noqa: E402
from four_bits_util import Cache4  # noqa: E402
from gpu_util import Guarded, stream  # noqa: E402

FP16, INT8, FP8, INT4 = cg.KV_FP16, cg.KV_INT8, cg.KV_FP8, cg.KV_INT4


def make(lens, dtype, **kw):
    if dtype == INT4:
        kw["block"] = max(32, kw.get("block", 32))
        return Cache4(lens, **kw)
    return Cache(lens, dtype=dtype, **kw)


def scores_of(c, seed=1, ties=True):
    s = torch.rand(c.pages, c.heads, c.page, generator=torch.Generator().manual_seed(seed)) ** 8
    return ((s * 64).round() / 64 if ties else s).cuda()


def kept(c, i, h, scores, budget, first, last):
    """Positions of sequence i that key head h keeps: sorted by score from the top, the lower position first."""
    n = max(0, c.lens[i])
    there = [t for t in range(n) if c.page_of(i, t) is not None]
    if len(there) <= budget:
        return there
    always = [t for t in there if t < first or t >= n - last]
    others = [t for t in there if first <= t < n - last]
    s = {t: float(scores[c.page_of(i, t), h, t % c.page]) for t in others}
    s = {t: -math.inf if math.isnan(x) else x for t, x in s.items()}
    order = sorted(others, key=lambda t: (math.isnan(float(scores[c.page_of(i, t), h, t % c.page])), -s[t], t))
    return sorted(always + order[:budget - len(always)])


def evict(c, to, scores, budget, first=0, last=0, max_kv=None, shift=None, to_scores=True):
    d = cg.EvictDesc.make(budget, keep_first=first, keep_last=last, max_kv=max_kv or max(1, max(c.lens)))
    ws, n = workspace(cg.codegemm_kv_evict_workspace_bytes(c.struct(), d))
    B = len(c.lens)
    guards = [Guarded(4 * B + (-4 * B) % 16), Guarded(4 * B + (-4 * B) % 16), Guarded(to.pages * c.heads * c.page * 4)]
    lens, shifts = (g.t[:4 * B].view(torch.int32).fill_(-9) for g in guards[:2])
    new = guards[2].view(torch.float32, (to.pages, c.heads, c.page)).fill_(-7.0)
    given = None if shift is None else torch.tensor(shift, dtype=torch.int32, device="cuda")
    cg.codegemm_kv_evict(c.struct(), to.struct(), d, scores, given, new if to_scores else None, lens, shifts, ws, n, stream())
    assert all(g.intact() for g in guards) and c.intact() and to.intact() and counters_are_clear()
    return lens, shifts, new


def raw(c, i, t, values):
    """A token's bits: codes, and what scales it (not of blocks)."""
    if isinstance(c, Cache4):
        return c.raw(i, t, values)
    return (c.place(c.v if values else c.k, i, t, values),)


def bits(x):
    return torch.empty(x.shape, dtype=x.dtype, device=x.device).copy_(x).view(torch.uint8)


def run(c, budget, first=0, last=0, scores=None, max_kv=None, shift=None, to=None, spare_to=None):
    scores = scores_of(c) if scores is None else scores
    lens = [min(budget, sum(c.page_of(i, t) is not None for t in range(max(0, n)))) for i, n in enumerate(c.lens)]
    kw = dict(heads=c.heads, dim=c.dim, page=c.page, block=c.block, seed=99, filled=[0] * len(lens))
    to = to or make(lens, c.dtype, **kw)
    if spare_to:
        spare_to(to)
    start = [x.clone() for x in (c.k, c.v, scores)]
    old = [None if x is None else x.clone() for x in (to.k, to.k_scales, to.v, to.v_scales)]
    got_lens, got_shift, new = evict(c, to, scores, budget, first, last, max_kv, shift)
    assert got_lens.tolist() == lens
    assert got_shift.tolist() == [(shift or [0] * len(lens))[i] + max(0, n) - m for i, (n, m) in enumerate(zip(c.lens, lens))]
    assert torch.equal(start[0].view(torch.uint8), c.k.view(torch.uint8)) and torch.equal(start[1].view(torch.uint8), c.v.view(torch.uint8)) and torch.equal(start[2].view(torch.int32), scores.view(torch.int32))
    expect_scores = torch.full_like(new, -7.0)
    for values in (False, True):
        pool, scales = (old[2], old[3]) if values else (old[0], old[1])
        mine, mine_s = (to.v, to.v_scales) if values else (to.k, to.k_scales)
        for i, m in enumerate(lens):
            stay = [kept(c, i, h, scores, budget, first, last) for h in range(c.heads)]
            assert all(len(s) == m for s in stay)
            for t in range(m):
                if to.page_of(i, t) is None:
                    continue
                for h in range(c.heads):
                    s = stay[h][t]
                    a, b = [x[h] for x in raw(c, i, s, values)], [x[h] for x in raw(to, i, t, values)]
                    if c.dtype in (FP16, INT4) or c.block == 1:
                        assert all(torch.equal(bits(x), bits(y)) for x, y in zip(a, b)), (values, i, t, h)
                    else:
                        b0 = t // c.block * c.block
                        was = [c.scale_of(c.v_scales if values else c.k_scales, i, stay[h][u])[h] for u in range(b0, min(b0 + c.block, m))]
                        now = to.scale_of(mine_s, i, t)[h]
                        assert float(now) == max(float(x) for x in was)
                        old_s = was[t - b0]
                        if float(old_s) == float(now):
                            assert torch.equal(a[0].contiguous(), b[0].contiguous())
                        else:
                            x = c.value(a[0].contiguous()) * (old_s / now).double()
                            half = 0.5 if c.dtype == INT8 else x.abs() * 2.0 ** -4 + 2.0 ** -10
                            assert bool(((to.value(b[0].contiguous()) - x).abs() <= half + 2.0 ** -17).all())
                    if not values:
                        expect_scores[to.page_of(i, t), h, t % to.page] = scores[c.page_of(i, s), h, s % c.page]
                # what is a token's may be anything that was checked; all else is as it was
                if isinstance(to, Cache4):
                    to.accept(pool, scales, i, t, values)
                else:
                    to.place(pool, i, t, values).copy_(to.place(mine, i, t, values))
                    if scales is not None:
                        to.scale_of(scales, i, t).copy_(to.scale_of(mine_s, i, t))
                        if c.block == 1:
                            for h in range(c.heads):
                                assert float(to.scale_of(mine_s, i, t)[h]) == float(c.scale_of(c.v_scales if values else c.k_scales, i, stay[h][t])[h])
        assert torch.equal(pool.view(torch.uint8), mine.view(torch.uint8)), "a place that is no token's was written"
        if scales is not None:
            assert torch.equal(scales.view(torch.int16), mine_s.view(torch.int16))
    assert torch.equal(expect_scores.view(torch.int32), new.view(torch.int32))          # NaN too
    return to


TYPES = [(FP16, 1), (INT8, 1), (INT8, 4), (INT8, 16), (FP8, 2), (FP8, 16), (INT4, 32)]


@pytest.mark.parametrize("dtype,block", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 256])
def test_types_and_dims(dtype, block, dim):
    run(make([70, 3, 0, 33], dtype, heads=2, dim=dim, block=block, seed=dim), 21, 2, 5)


@pytest.mark.parametrize("dim", [16, 48, 80])
@pytest.mark.parametrize("dtype", [FP16, INT8, FP8])
def test_dims_that_four_bits_have_not(dtype, dim):
    run(make([40, 17], dtype, heads=3, dim=dim, block=4, seed=dim), 18)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [FP16, INT8, INT4])
def test_pages(page, dtype):
    run(make([300, 17, 200], dtype, heads=1, dim=64, page=page, block=16), 130, 4, 20)


@pytest.mark.parametrize("block", [32, 64, 128, 256])
def test_long_blocks(block):
    run(make([600, 250], INT8, heads=1, dim=64, page=256, block=block), 270, 1, 9)


@pytest.mark.parametrize("budget,first,last", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (2, 1, 1), (16, 0, 0), (17, 0, 17), (50, 50, 0), (50, 20, 30), (69, 0, 0), (70, 3, 3), (1 << 30, 5, 5),
                                               (1 << 30, 0, 1 << 30)])
def test_budgets(budget, first, last):
    run(make([70, 3, 0, 33, 1], INT4, heads=2, dim=64), budget, first, last)


def test_scores_that_are_equal_or_none():
    c = make([100, 65], FP16, heads=2, dim=32)
    for x in (0.0, -0.0, 1.0, float("inf"), float("-inf"), float("nan"), -3.0):
        run(c, 33, 1, 2, scores=torch.full((c.pages, 2, 16), x, device="cuda"))
    s = scores_of(c)
    odd = [float("nan"), float("inf"), float("-inf"), -0.0, 0.0, -1.0, 1e-40, -1e-40, 3e38, 1e-45]
    g = torch.Generator().manual_seed(3)
    s.copy_(torch.tensor(odd)[torch.randint(0, len(odd), s.shape, generator=g)].cuda())
    for budget in (5, 20, 40, 64, 90):
        run(c, budget, 0, 0, scores=s)
    run(c, 40, scores=scores_of(c, ties=False) * -1)


def test_pages_that_are_not_there():
    c = make([100, 64, 40], INT4, heads=2, dim=64, page=16)
    c.table[0, 2] = -1
    c.table[1, :] = c.pages + 1
    c.table[2, 0] = -4
    c.table_dev.copy_(c.table.cuda())
    run(c, 50, 3, 10)

    def absent(to):
        to.table[0, 1] = -1
        to.table[2, 0] = to.pages
        to.table_dev.copy_(to.table.cuda())
    for dtype in (INT4, INT8, FP16):
        run(make([100, 64, 40], dtype, heads=2, dim=64, page=16, block=4), 50, 3, 10, spare_to=absent)


def test_lengths_beyond_the_table_and_below_zero():
    c = make([64, 48, 0], INT4, heads=1, dim=64, page=16, max_pages=4)
    c.lens_dev.copy_(torch.tensor([100, 48, -5], dtype=torch.int32))
    to = make([20, 20, 0], INT4, heads=1, dim=64, page=16, seed=99, filled=[0, 0, 0])
    scores = scores_of(c)
    lens, shift, _ = evict(c, to, scores, 20, 0, 10)
    assert lens.tolist() == [20, 20, 0] and shift.tolist() == [80, 28, 0]
    # the last 10 of 100 have no page; so the best 20 of the 64 that have
    stay = kept(c, 0, 0, scores, 20, 0, 0)
    for t in range(20):
        assert all(torch.equal(x, y) for x, y in zip(c.raw(0, stay[t], False), to.raw(0, t, False)))


@pytest.mark.parametrize("dtype", [FP16, INT4])
def test_shift_and_hints(dtype):
    c = make([150, 40, 9], dtype, heads=2, dim=64)
    run(c, 30, 2, 4, shift=[5, 0, 1000], max_kv=1)
    run(c, 30, 2, 4, shift=[5, 0, 1000], max_kv=(1 << 31) - 1)


def big(lens, dim=64, heads=1, page=64, seed=1):
    c = Cache4(lens, heads=heads, dim=dim, page=page, seed=seed)
    return c


@pytest.mark.parametrize("n,budget", [(40000, 39999), (40000, 10000), (33000, 100), (70001, 32768), (5000, 4096)])
def test_long(n, budget):
    """More scores than LDS holds, more than a wavefront's stretch; positions against a sort."""
    c = big([n, 100])
    scores = torch.rand(c.pages, 1, c.page, generator=torch.Generator().manual_seed(4)).cuda()
    scores = (scores ** 8 * 4096).round() / 4096                       # ties in their thousands
    lens = [budget, min(100, budget)]
    to = Cache4(lens, heads=1, dim=64, page=64, seed=7, filled=[0, 0])
    got_lens, _, new = evict(c, to, scores, budget, 7, 50)
    assert got_lens.tolist() == lens
    t = torch.arange(n, device="cuda")
    s = scores[c.table[0].long().cuda()[t // 64], 0, t % 64]
    s = torch.where((t < 7) | (t >= n - 50), torch.inf, s)
    want = torch.sort(s, descending=True, stable=True).indices[:budget].sort().values
    u = torch.arange(budget, device="cuda")
    src, dst = c.table[0].long().cuda()[want // 64], to.table[0].long().cuda()[u // 64]
    assert torch.equal(new[dst, 0, u % 64], scores[src, 0, want % 64])
    assert torch.equal(to.k[dst, 0, u % 64], c.k[src, 0, want % 64]) and torch.equal(to.k_scales[dst, 0, u % 64], c.k_scales[src, 0, want % 64])
    k0, v0, _ = c.sequence(0, 0, n)
    k1, v1, _ = to.sequence(0, 0, budget)
    assert torch.equal(k0[want], k1) and torch.equal(v0[want], v1)


def test_nan_scales():
    """A NaN scale makes its new block NaN; other blocks are as they are."""
    c = make([64], INT8, heads=1, dim=32, block=4)
    c.scale_of(c.k_scales, 0, 20).fill_(float("nan"))
    to = make([40], INT8, heads=1, dim=32, block=4, seed=9, filled=[0])
    scores = scores_of(c, ties=False)
    evict(c, to, scores, 40)
    stay = kept(c, 0, 0, scores, 40, 0, 0)
    for t in range(40):
        mine = [stay[u] for u in range(t // 4 * 4, min(40, t // 4 * 4 + 4))]
        assert bool(to.scale_of(to.k_scales, 0, t).isnan().all()) == any(20 <= u < 24 for u in mine)


def test_one_pool_one_array_one_set_of_lengths_and_a_graph():
    """`to` in other pages of the same pool, scores in the same array, lengths and shifts where they were: eager and replayed."""
    lens = [90, 33, 60]

    def build():
        c = Cache4(lens, heads=2, dim=64, page=16, seed=2, spare=12)
        used = set(c.table.flatten().tolist())
        free = [p for p in range(c.pages) if p not in used]
        table = torch.full((3, c.max_pages), -1, dtype=torch.int32)
        for i, m in enumerate((40, 33, 40)):
            for j in range(-(-m // 16)):
                table[i, j] = free.pop()
        to_table = table.cuda()
        to = cg.KvCache.make(c.k, c.v, c.k_scales, c.v_scales, to_table, c.lens_dev, kv_heads=2, head_dim=64, num_pages=c.pages, page_size=16, dtype=INT4, scale_block=32,
                             num_seqs=3, max_pages=c.max_pages)
        return c, to, to_table, scores_of(c), torch.tensor([3, 0, 0], dtype=torch.int32, device="cuda")

    d = cg.EvictDesc.make(40, keep_first=2, keep_last=8, max_kv=90)
    results = []
    for graphed in (False, True):
        c, to, table, scores, shift = build()
        keep = (table,)
        ws = torch.zeros(cg.codegemm_kv_evict_workspace_bytes(c.struct(), d), dtype=torch.uint8, device="cuda")

        def call():
            cg.codegemm_kv_evict(c.struct(), to, d, scores, shift, scores, c.lens_dev, shift, ws, ws.numel(), stream())
        for again in range(3):
            c.lens_dev.copy_(torch.tensor(lens, dtype=torch.int32))
            if graphed:
                if again == 0:
                    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
                    torch.cuda.synchronize()
                    with torch.cuda.graph(graph, stream=side):
                        call()
                graph.replay()
            else:
                call()
            torch.cuda.synchronize()
            results.append([x.clone() for x in (c.k, c.k_scales, c.v, c.v_scales, scores, c.lens_dev, shift)])
        assert keep
    assert results[0][5].tolist() == [40, 33, 40] and results[0][6].tolist() == [53, 0, 20] and results[2][6].tolist() == [153, 0, 60]
    for a, b in zip(results[:3], results[3:]):
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))

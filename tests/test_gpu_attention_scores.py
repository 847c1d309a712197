"""codegemm_attn_scores and codegemm_attn_decode_scores against their definition in 64 bits: softmax weights summed per cached token and key head."""
import pytest
import torch

pytestmark = pytest.mark.gpu

cg = pytest.importorskip("paper_2512_17970_amd")
from attention_util import Cache, check, counters_are_clear, decode_exact, starts, workspace  # noqa: E402
from four_bits_util import Cache4  # noqa: E402
from gpu_util import Guarded, stream  # noqa: E402

FP16, INT8, FP8, INT4 = cg.KV_FP16, cg.KV_INT8, cg.KV_FP8, cg.KV_INT4


def make(lens, dtype, **kw):
    if dtype == INT4:
        kw.pop("block", None)
        return Cache4(lens, **kw)
    kw.pop("quick", None)
    return Cache(lens, dtype=dtype, **kw)


def sequence(c, i, lo, hi):
    """keys [hi - lo][heads][dim] in 64 bits, and which of them have a page"""
    if isinstance(c, Cache4):
        k, _, seen = c.sequence(i, lo, hi)
        return k, seen
    rows = [c.read(i, t, False) for t in range(lo, hi)]
    zero = torch.zeros(c.heads, c.dim, dtype=torch.float64, device="cuda")
    return torch.stack([zero if x is None else x for x in rows]) if rows else zero[None][:0], torch.tensor([x is not None for x in rows], dtype=torch.bool, device="cuda")


def exact(c, q, new, window=0, scale=None, lens=None):
    """Per sequence the sums [heads][n] in 64 bits and a bound on their error.  A score has up to D + 4 roundings (2^-24) of the sum of its products' sizes, its
    weight the same of 1, plus what exponential and sums in 32 bits add: some 4 + log2(n) and the row's sum, whose own scores are off alike."""
    out, at = [], 0
    D, Hq = q.shape[2], q.shape[1]
    r = Hq // c.heads
    scale = D ** -0.5 if scale is None else scale
    for i, rows in enumerate(new):
        n = max(0, (lens or c.lens)[i])
        k, paged = sequence(c, i, 0, n)
        sums, bound = (torch.zeros(c.heads, n, dtype=torch.float64, device="cuda") for _ in range(2))
        t = torch.arange(n, device="cuda")
        for j in range(rows):
            p = n - rows + j
            seen = paged & (t <= p) & ((t > p - window) if window else True)
            if p < 0 or not bool(seen.any()):
                continue
            for h in range(Hq):
                kh = k[:, h // r]
                x = q[at + j, h].double()
                s = torch.where(seen, (kh * x).nan_to_num().sum(-1) * scale, -torch.inf)
                w = torch.softmax(s, 0)
                size = float(((kh * x).nan_to_num().abs().sum(-1) * abs(scale))[seen].max())
                sums[h // r] += w
                bound[h // r] += w * (2 * (D + 4) * size + 16 + n / 64) * 2.0 ** -24
        at += rows
        bound += sums * (rows * r + 4) * 2.0 ** -24 + 2.0 ** -60
        out.append((sums, bound, paged))
    return out


def run(c, q, new, *, window=0, scale=None, max_kv=None, first=None, earlier=True, in_place=False, single=False, cu=True, q_stride=0):
    """One call; checks every place of `scores` and returns (scores, out)."""
    B, (T, Hq, D) = len(new), q.shape
    desc = cg.AttnDesc.make(Hq, c.heads, D, num_seqs=B, total_q=T, max_kv=max_kv or max(1, max(c.lens)), scale=D ** -0.5 if scale is None else scale, window=window, q_stride=q_stride)
    s = c.struct()
    shape = (c.pages, c.heads, c.page)
    before = torch.rand(shape, generator=torch.Generator().manual_seed(5)).cuda() * 3
    guard = Guarded(before.numel() * 4)
    scores = guard.view(torch.float32, shape)
    scores.copy_(before if in_place else torch.full_like(before, -7.0))
    was = scores.clone()
    had = scores if in_place else before if earlier else None
    firsts = None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda")
    out = None
    if single:
        og = Guarded(T * Hq * D * 2)
        out = og.view(torch.float16, (T, Hq, D)).fill_(float("nan"))
        ws, n = workspace(cg.codegemm_attn_decode_scores_workspace_bytes(s, desc))
        cg.codegemm_attn_decode_scores(s, desc, q, out, firsts, had, scores, ws, n, stream())
        assert og.intact()
    else:
        ws, n = workspace(cg.codegemm_attn_scores_workspace_bytes(s, desc))
        cg.codegemm_attn_scores(s, desc, q, starts(new) if cu else None, firsts, had, scores, ws, n, stream())
    assert guard.intact() and c.intact() and counters_are_clear()
    expect = was.clone()
    for i, (sums, bound, paged) in enumerate(exact(c, q if not q_stride else q, new, window, scale)):
        n = sums.shape[1]
        lo = n - new[i] if first is None else first[i]
        for t in range(n):
            if not bool(paged[t]):
                continue
            at = (c.page_of(i, t), slice(None), t % c.page)
            want = sums[:, t] + (before[at].double() if (earlier or in_place) and t < lo else 0)
            err = (scores[at].double() - want).abs()
            assert bool((err <= bound[:, t] + 2.0 ** -23 * want.abs()).all()), f"token {t} of {i}: {float((err / (bound[:, t] + 2.0 ** -23 * want.abs())).max()):.2f} times the bound"
            expect[at] = scores[at]
    assert torch.equal(expect, scores), "a place that is no token's was written"
    return scores, out


def queries(T, Hq, D, seed=1, size=1.5):
    return (torch.randn(T, Hq, D, generator=torch.Generator().manual_seed(seed)) * size).half().cuda()


TYPES = [(FP16, 1), (INT8, 1), (INT8, 4), (INT8, 16), (FP8, 2), (FP8, 16), (INT4, 32)]


@pytest.mark.parametrize("dtype,block", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 256])
def test_types_and_dims(dtype, block, dim):
    c = make([70, 3, 0, 33], dtype, heads=2, dim=dim, block=block, seed=dim)
    run(c, queries(6, 6, dim), [3, 1, 0, 2])
    run(c, queries(4, 6, dim), [1, 1, 1, 1], single=True)


@pytest.mark.parametrize("dim", [16, 48, 80, 144])
@pytest.mark.parametrize("dtype", [FP16, INT8, FP8])
def test_dims_that_four_bits_have_not(dtype, dim):
    run(make([40, 17], dtype, heads=1, dim=dim, block=4, seed=dim), queries(5, 3, dim), [4, 1])


@pytest.mark.parametrize("heads,group", [(1, 1), (3, 5), (1, 16), (1, 17), (2, 8), (1, 130)])
@pytest.mark.parametrize("single", [False, True])
def test_heads(heads, group, single):
    c = make([50, 21], INT4, heads=heads, dim=64)
    run(c, queries(2, heads * group, 64), [1, 1], single=single, cu=not single)
    run(c, queries(2, heads * group, 64), [1, 1], cu=False)


@pytest.mark.parametrize("window", [0, 1, 5, 33, 100, (1 << 31) - 1])
@pytest.mark.parametrize("new", [[1, 1, 1], [20, 5, 40]])
@pytest.mark.parametrize("dtype", [FP16, INT4])
def test_windows_and_queries(window, new, dtype):
    c = make([90, 5, 47], dtype, heads=2, dim=64, page=16)
    run(c, queries(sum(new), 4, 64), new, window=window)
    if max(new) == 1:
        run(c, queries(3, 4, 64), new, window=window, single=True)


@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_pages_that_are_not_there(page):
    c = make([300, 90, 16, 40], INT4, heads=2, dim=64, page=page, seed=4)
    c.table[0, 0] = -1
    c.table[1, :] = c.pages
    c.table_dev.copy_(c.table.cuda())
    run(c, queries(9, 4, 64), [4, 3, 1, 1])
    run(c, queries(4, 4, 64), [1, 1, 1, 1], single=True)


@pytest.mark.parametrize("kw", [dict(earlier=False), dict(in_place=True), dict(first=[0, 0, 0]), dict(first=[10, 1000, -5]), dict(first=[7, 3, 2], in_place=True), dict(first=[9, 9, 9], earlier=False)])
def test_what_they_had_before(kw):
    c = make([70, 5, 40], INT8, heads=2, dim=64, block=16)
    run(c, queries(12, 4, 64), [6, 2, 4], **kw)
    run(c, queries(3, 4, 64), [1, 1, 1], single=True, **kw)


def test_more_queries_than_tokens_and_idle_slots():
    c = make([3, 0, 20, 0], INT4, heads=2, dim=64)
    run(c, queries(12, 4, 64), [5, 2, 4, 1])
    run(c, queries(4, 4, 64), [1, 1, 1, 1], single=True)
    c = make([3, -2], INT4, heads=2, dim=64)
    run(c, queries(3, 4, 64), [2, 1])


@pytest.mark.parametrize("window", [0, 5])
def test_the_largest_length(window):
    """Of 2^31 - 1 tokens the table holds 64: rows without a window see them all, rows with one stand behind."""
    c = make([64, 40], INT8, heads=1, dim=64, page=16, max_pages=4)
    c.lens_dev.copy_(torch.tensor([2 ** 31 - 1, 40], dtype=torch.int32))
    q = queries(6, 4, 64)
    desc = cg.AttnDesc.make(4, 1, 64, num_seqs=2, total_q=6, max_kv=64, scale=0.125, window=window)
    s = c.struct()
    ws, n = workspace(cg.codegemm_attn_scores_workspace_bytes(s, desc))
    scores = torch.full((c.pages, 1, 16), -7.0, device="cuda")
    cg.codegemm_attn_scores(s, desc, q, starts([3, 3]), None, None, scores, ws, n, stream())
    got = torch.stack([scores[c.page_of(0, t), 0, t % 16] for t in range(64)])
    if window:
        assert bool((got == 0).all())
    else:
        assert bool((got > 0).all()) and abs(float(got.double().sum()) - 12) < 1e-3
    other = torch.stack([scores[c.page_of(1, t), 0, t % 16] for t in range(40)])
    assert abs(float(other.double().sum()) - 12) < 1e-3


def test_lengths_beyond_the_table():
    """The last places of the table are the last that count; queries stand behind them."""
    c = make([64, 40], INT4, heads=1, dim=64, page=16, max_pages=4)
    c.lens_dev.copy_(torch.tensor([100, 40], dtype=torch.int32))
    q = queries(2, 4, 64)
    desc = cg.AttnDesc.make(4, 1, 64, num_seqs=2, total_q=2, max_kv=64, scale=0.125)
    s = c.struct()
    ws, n = workspace(cg.codegemm_attn_scores_workspace_bytes(s, desc))
    scores = torch.zeros(c.pages, 1, 16, device="cuda")
    cg.codegemm_attn_scores(s, desc, q, None, None, None, scores, ws, n, stream())
    for i, (sums, bound, _) in enumerate(exact(c, q, [1, 1])):             # (position 99 sees all 64)
        got = torch.stack([scores[c.page_of(i, t), :, t % 16] for t in range(c.lens[i])], dim=1)
        assert bool(((got.double() - sums).abs() <= bound + 2.0 ** -23 * sums).all())


@pytest.mark.parametrize("dtype,dim", [(INT4, 128), (INT8, 64), (FP16, 128), (INT4, 256)])
def test_long_and_many_queries(dtype, dim):
    """Several blocks of keys to a workgroup, several groups of rows, lengths that the host does not know; the same bits again."""
    c = make([1500, 300], dtype, heads=1, dim=dim, block=16, page=64, quick=True)
    q = queries(70, 8, dim)
    a, _ = run(c, q, [40, 30])
    b, _ = run(c, q, [40, 30], max_kv=1)
    again, _ = run(c, q, [40, 30])
    assert torch.equal(a, again)
    single = queries(2, 8, dim)
    a, _ = run(c, single, [1, 1], single=True)
    b, _ = run(c, single, [1, 1], single=True, max_kv=1)


def test_sums_are_what_was_given_out():
    """Every row gives out 1 in all, whatever the scores: large, equal, negative scale."""
    c = make([500, 64], INT4, heads=2, dim=64, page=64)
    for scale, size in ((None, 1.5), (0.0, 1.0), (-1.0, 1.0), (3.0, 30.0), (1e20, 1.0)):
        q = queries(9, 8, 64, size=size)
        desc = cg.AttnDesc.make(8, 2, 64, num_seqs=2, total_q=9, max_kv=500, scale=0.125 if scale is None else scale)
        s = c.struct()
        ws, n = workspace(cg.codegemm_attn_scores_workspace_bytes(s, desc))
        scores = torch.zeros(c.pages, 2, 64, device="cuda")
        cg.codegemm_attn_scores(s, desc, q, starts([4, 5]), None, None, scores, ws, n, stream())
        for i, rows in enumerate((4, 5)):
            got = sum(scores[c.page_of(i, t), :, t % 64].double() for t in range(c.lens[i]))
            assert bool(((got - rows * 4).abs() <= rows * 4 * (c.lens[i] + 64) * 2.0 ** -24).all())
        single = queries(2, 8, 64, size=size)
        desc = cg.AttnDesc.make(8, 2, 64, num_seqs=2, total_q=2, max_kv=500, scale=0.125 if scale is None else scale)
        ws, n = workspace(cg.codegemm_attn_decode_scores_workspace_bytes(s, desc))
        cg.codegemm_attn_decode_scores(s, desc, single, torch.empty_like(single), None, None, scores.zero_(), ws, n, stream())
        for i in range(2):
            got = sum(scores[c.page_of(i, t), :, t % 64].double() for t in range(c.lens[i]))
            assert bool(((got - 4).abs() <= 4 * (c.lens[i] + 64) * 2.0 ** -24).all())


@pytest.mark.parametrize("size", [1e-3, 1.0, 8.0, 40.0, 600.0])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("dim", [64, 128])
def test_rows_whose_scores_are_all_far_from_zero(size, sign, dim):
    """Keys that point one way, queries along it and against it: all scores of a row lie near sign * size * 8 (up to 4800 and more), on one side of what exp2 holds as on the
    other; some rows small beside them."""
    for new in ([40, 3], [1, 1]):
        c = make([700, 90], FP16, heads=1, dim=dim, page=64)
        g = torch.Generator().manual_seed(2)
        c.k.copy_((1 + 0.02 * torch.randn(c.k.shape, generator=g)).half().cuda())
        q = (sign * size * 8 / dim ** 0.5 * (1 + 0.1 * torch.rand(sum(new), 4, dim, generator=g))).half().cuda()
        q[::3] *= 0.01
        run(c, q, new)
        if max(new) == 1:
            run(c, q, new, single=True)


@pytest.mark.parametrize("dtype,block", TYPES)
def test_the_attention_beside_them(dtype, block):
    lens = [700, 3, 0, 64, 257]
    c = make(lens, dtype, heads=2, dim=64, block=block, page=32)
    q = queries(5, 8, 64)
    _, out = run(c, q, [1] * 5, single=True, window=0)
    if dtype == INT4:
        from test_gpu_four_bits import decode, decode_exact as exact4
        check(out, *exact4(c, q), "out")
        assert torch.equal(out, decode(c, q))
    else:
        from attention_util import decode
        check(out, *decode_exact(c, q), "out")
        if dtype != FP16:
            assert torch.equal(out, decode(c, q))


def test_nan_keys_stay_with_those_who_see_them():
    c = make([40, 40], FP16, heads=1, dim=64)
    c.place(c.k, 0, 30, False).fill_(float("nan"))
    q = queries(20, 2, 64)
    desc = cg.AttnDesc.make(2, 1, 64, num_seqs=2, total_q=20, max_kv=40, scale=0.125)
    s = c.struct()
    ws, n = workspace(cg.codegemm_attn_scores_workspace_bytes(s, desc))
    scores = torch.zeros(c.pages, 1, 16, device="cuda")
    cg.codegemm_attn_scores(s, desc, q, starts([10, 10]), None, None, scores, ws, n, stream())
    got = torch.stack([scores[c.page_of(1, t), 0, t % 16] for t in range(40)])
    assert bool(got.isfinite().all()) and abs(float(got.double().sum()) - 20) < 1e-4
    # the first sequence: queries stand at 30 and on, so all see the key
    assert bool(torch.stack([scores[c.page_of(0, t), 0, t % 16] for t in range(31)]).isnan().all())
    desc = cg.AttnDesc.make(2, 1, 64, num_seqs=2, total_q=20, max_kv=40, scale=0.125, window=3)
    cg.codegemm_attn_scores(s, desc, q, starts([10, 10]), None, None, scores.zero_(), ws, n, stream())
    got = torch.stack([scores[c.page_of(0, t), 0, t % 16] for t in range(40)])
    assert bool((got[:28] == 0).all()) and bool(got[28:33].isnan().all()) and bool(got[35:].isfinite().all())


@pytest.mark.parametrize("new", [[1, 1], [9, 33]])
def test_infinite_keys_that_all_rows_turn_away_from(new):
    """A key of infinite length whose scores are -inf has no weight, and does not touch its neighbours', however many rows there are."""
    c = make([200, 400], FP16, heads=2, dim=128, page=64, seed=12)
    q = queries(sum(new), 6, 128)
    q[..., 7] = -q[..., 7].abs() - 0.5
    for t in (3, 100, 130):
        page, slot = c.page_of(1, t), t % 64
        c.k[page, :, slot, 7] = float("inf")
    s = c.struct()
    desc = cg.AttnDesc.make(6, 2, 128, num_seqs=2, total_q=sum(new), max_kv=400, scale=128 ** -0.5)
    scores = torch.full((c.pages, 2, 64), -7.0, device="cuda")
    if new == [1, 1]:
        ws, n = workspace(cg.codegemm_attn_decode_scores_workspace_bytes(s, desc))
        cg.codegemm_attn_decode_scores(s, desc, q, torch.empty_like(q), None, None, scores, ws, n, stream())
    else:
        ws, n = workspace(cg.codegemm_attn_scores_workspace_bytes(s, desc))
        cg.codegemm_attn_scores(s, desc, q, starts(new), None, None, scores, ws, n, stream())
    for i in range(2):
        got = torch.stack([scores[c.page_of(i, t), :, t % 64] for t in range(c.lens[i])])
        assert bool(got.isfinite().all())
        # (weights are rounded to 24 bits a few times each; 2^-16 is far above that)
        assert bool((got.double().sum(0) - 3 * new[i]).abs().max() < 3 * new[i] * 2.0 ** -16)
        if i == 1:
            assert bool((got[[3, 100, 130]] == 0).all())


def test_strides_streams_and_graphs():
    c = make([100, 257], INT4, heads=2, dim=128, page=32, seed=6)
    q = queries(2, 8, 128)
    wide = torch.zeros(2, 8 * 128 + 64, dtype=torch.float16, device="cuda")
    wide[:, :1024] = q.view(2, -1)
    want, out = run(c, q, [1, 1], single=True, earlier=False)
    s = c.struct()
    desc = cg.AttnDesc.make(8, 2, 128, num_seqs=2, total_q=2, max_kv=257, scale=128 ** -0.5, q_stride=wide.shape[1])
    ws = torch.zeros(cg.codegemm_attn_decode_scores_workspace_bytes(s, desc), dtype=torch.uint8, device="cuda")
    got, o = torch.full_like(want, -7.0), torch.empty_like(out)

    def call():
        cg.codegemm_attn_decode_scores(s, desc, wide, o, None, None, got, ws, ws.numel(), stream())
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(o, out)
    with torch.cuda.graph(graph, stream=side):
        call()
    for n in (257, 100, 1, 200):
        c.lens_dev[1] = n
        got.fill_(-7.0)
        call()
        torch.cuda.synchronize()
        eager, eager_o = got.clone(), o.clone()
        got.fill_(-7.0)
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, eager) and torch.equal(o, eager_o)

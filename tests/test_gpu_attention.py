"""codegemm_attn_decode and codegemm_attn_prompt against their definitions in 64 bits, at the sizes, masks and contents where they can go wrong."""
import pytest
import torch

pytestmark = pytest.mark.gpu

cg = pytest.importorskip("paper_2512_17970_amd")
from attention_util import Cache, check, counters_are_clear, decode, decode_exact, prompt, prompt_exact, starts, workspace  # noqa: E402
from gpu_util import stream  # noqa: E402

FP16, INT8, FP8 = cg.binding.KV_FP16, cg.binding.KV_INT8, cg.binding.KV_FP8
LENS = [0, 1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 130, 300]


def queries(B, Hq, D, seed=1, size=1.5):
    return (torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(seed)) * size).half().cuda()


# ---- single tokens over the cache ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,block", [(FP16, 1), (INT8, 1), (INT8, 2), (INT8, 4), (INT8, 8), (INT8, 16), (FP8, 1), (FP8, 16)])
@pytest.mark.parametrize("dim", [16, 64, 80, 128, 208, 256])
def test_decode_types_and_lengths(dtype, block, dim):
    c = Cache(LENS, heads=2, dim=dim, dtype=dtype, block=block, seed=dim + block)
    q = queries(len(LENS), 6, dim)
    got = decode(c, q)
    check(got, *decode_exact(c, q), f"type {dtype} block {block} D {dim}")
    assert not bool(got[0].any()), "a sequence without tokens"


@pytest.mark.parametrize("page,block", [(16, 16), (32, 32), (64, 16), (128, 128), (256, 64), (256, 256)])
@pytest.mark.parametrize("dtype", [INT8, FP8])
def test_decode_pages_and_blocks(page, block, dtype):
    c = Cache([1, 255, 256, 257, 600], heads=1, dim=128, page=page, dtype=dtype, block=block, seed=page + block)
    q = queries(5, 8, 128)
    check(decode(c, q), *decode_exact(c, q), f"page {page} block {block}")


@pytest.mark.parametrize("heads,group", [(1, 1), (3, 5), (1, 16), (2, 17), (1, 33), (5, 7)])
def test_decode_head_layouts(heads, group):
    c = Cache([70, 200], heads=heads, dim=64, dtype=INT8, block=16, seed=heads)
    q = queries(2, heads * group, 64)
    check(decode(c, q), *decode_exact(c, q), f"{heads} x {group}")


@pytest.mark.parametrize("window", [1, 15, 16, 64, 100, 1 << 30])
@pytest.mark.parametrize("dtype,block", [(FP16, 1), (INT8, 4), (FP8, 16)])
def test_decode_window(window, dtype, block):
    c = Cache([0, 1, 16, 99, 100, 101, 350], heads=1, dim=64, dtype=dtype, block=block, seed=window % 97)
    q = queries(7, 2, 64)
    check(decode(c, q, window=window), *decode_exact(c, q, window=window), f"window {window}")


@pytest.mark.parametrize("dtype,block", [(FP16, 1), (INT8, 1), (INT8, 16), (FP8, 16)])
def test_decode_tokens_without_a_page_do_not_count(dtype, block):
    c = Cache([200, 200, 40], heads=1, dim=64, dtype=dtype, block=block, seed=5)
    c.table[0, 3] = -1
    c.table[0, 12] = c.pages                       # the last one
    c.table[1, :] = 1 << 30                        # none at all
    c.table_dev.copy_(c.table)
    q = queries(3, 4, 64)
    got = decode(c, q)
    check(got, *decode_exact(c, q), "missing pages")
    assert not bool(got[1].any())


def test_decode_lengths_beyond_the_table_end_there():
    c = Cache([64, 64], heads=1, dim=64, dtype=INT8, block=16, seed=6)
    q = queries(2, 4, 64)
    want = decode_exact(c, q)
    c.lens_dev.copy_(torch.tensor([2 ** 31 - 1, 65], dtype=torch.int32))
    check(decode(c, q), *want, "lengths beyond the page table")
    c.lens_dev.fill_(-3)
    assert not bool(decode(c, q).any())


def test_decode_windows_beyond_the_table():
    """The last tokens of a length that the page table does not reach have no page: nothing is attended to."""
    c = Cache([64, 64, 64], heads=1, dim=64, dtype=INT8, block=16, seed=6)
    q = queries(3, 4, 64)
    c.lens_dev.copy_(torch.tensor([2 ** 31 - 1, 64 + 31, 64 + 40], dtype=torch.int32))
    assert not bool(decode(c, q, window=31).any())
    got, (want, bound) = decode(c, q, window=40), decode_exact(c, q, window=9)       # of the second, positions 55 to 63
    check(got[1], want[1], bound[1], "a window over the end")
    assert not bool(got[0].any()) and not bool(got[2].any())


@pytest.mark.parametrize("new,total", [([20], [700]), ([5, 70], [300, 70])])
def test_prompt_hints(new, total):
    """Any hint of the longest sequence."""
    q, k, v = packed(sum(new), sum(total), 4, 2, 64)
    for hint in (1, 2 ** 31 - 1):
        check(prompt(q, k, v, new, total, max_kv=hint), *prompt_exact(q, k, v, new, total), f"hint {hint}")


@pytest.mark.parametrize("dtype,block", [(FP16, 1), (INT8, 4), (INT8, 16), (FP8, 64)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_decode_split_ranges(dtype, block, dim):
    """Few sequences: their keys are split over workgroups and joined; the hint of the longest length does not change what is right."""
    lens = [1, 700, 1500, 2900]
    c = Cache(lens, heads=1, dim=dim, page=64, dtype=dtype, block=block, seed=9)
    q = queries(4, 8, dim)
    want = decode_exact(c, q)
    for hint in (1, 700, 2900, 1 << 20, 2 ** 31 - 1):
        got = decode(c, q, max_kv=hint)
        check(got, *want, f"hint {hint}")
        assert torch.equal(got, decode(c, q, max_kv=hint)), "bits differ from call to call"


@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("dtype,block", [(FP16, 1), (INT8, 4), (FP8, 16)])
def test_decode_more_items_than_compute_units(dtype, block, dim):
    """Two workgroups a unit; sequences of many lengths, more of them than a wavefront has lanes, some empty, one long enough to be cut."""
    lens = [(13 * i) % 40 for i in range(69)] + [1500]
    c = Cache(lens, heads=4, dim=dim, dtype=dtype, block=block, seed=dim)
    q = queries(70, 8, dim)
    got = decode(c, q)
    check(got, *decode_exact(c, q), f"type {dtype} D {dim}")
    assert torch.equal(got, decode(c, q))


def test_decode_strides_and_scale():
    c = Cache([100, 333], heads=2, dim=64, dtype=FP8, block=16, seed=11)
    wide = queries(2, 8, 64).reshape(2, 512).repeat(1, 2)[:, :640].contiguous()
    q = wide[:, 64:64 + 256]                       # four heads of a wider row
    out = torch.full((2, 400), 7.0, dtype=torch.float16, device="cuda")
    for scale in (0.05, -0.2, 0.0):
        d = cg.AttnDesc.make(4, 2, 64, num_seqs=2, total_q=2, max_kv=333, scale=scale, q_stride=640, out_stride=400)
        s = c.struct()
        ws, n = workspace(cg.codegemm_attn_decode_workspace_bytes(s, d))
        cg.codegemm_attn_decode(s, d, q, out, ws, n, stream())
        check(out[:, :256].reshape(2, 4, 64), *decode_exact(c, q.reshape(2, 4, 64), scale=scale), f"scale {scale}")
        assert bool((out[:, 256:] == 7.0).all())


def test_decode_extreme_scores_and_scales():
    """Scores far apart, one key far above all others late in the sequence, and value scales over twelve orders of magnitude."""
    c = Cache([400], heads=1, dim=64, dtype=INT8, block=1, seed=13)
    q = queries(1, 4, 64, size=20.0)
    check(decode(c, q, scale=1.0), *decode_exact(c, q, scale=1.0), "peaked")
    c.v_scales.copy_(torch.exp(torch.randn(c.v_scales.shape, generator=torch.Generator().manual_seed(3)) * 4 - 8).cuda())
    want, bound = decode_exact(c, q * 0.05)
    fine = want.abs() < 6e4
    got = decode(c, q * 0.05)
    check(torch.where(fine, got, 0), torch.where(fine, want, 0.0), bound, "value scales")
    c.k_scales.zero_()
    c.v_scales.zero_()
    assert not bool(decode(c, q).any()), "all scales zero"


def test_decode_nan_reaches_only_those_that_see_it():
    c = Cache([100, 100, 100], heads=2, dim=64, dtype=FP16, seed=15)
    c.place(c.v, 0, 50, True)[0, 7] = float("nan")
    c.place(c.k, 1, 3, False)[1, 9] = float("inf")
    q = queries(3, 4, 64)
    got = decode(c, q)
    want, bound = decode_exact(c, q)
    assert bool(got[0, :2, 7].isnan().all())
    got[0, :2, 7], want[0, :2, 7] = 0, 0
    finite = want.isfinite()                       # a score of -inf has no weight, one of +inf makes a NaN
    assert torch.equal(finite, got.isfinite())
    check(torch.where(finite, got, 0), torch.where(finite, want, 0.0), bound, "NaN and infinity")


def test_decode_pool_beyond_32_bits():
    """A pool of more than 2^32 bytes, the sequence's pages at its end."""
    heads, dim, page = 8, 128, 256
    pages = (1 << 32) // (heads * dim * page) + 9
    pool = [torch.empty(pages, heads, *shape, dtype=torch.uint8, device="cuda") for shape in ((page, dim), (page // 16, dim, 16))]
    small = Cache([700], heads=heads, dim=dim, page=page, dtype=INT8, block=64, seed=17)
    q = queries(1, 16, dim)
    want = decode_exact(small, q)
    scales = [torch.full((pages, heads, page // 64), float("nan"), device="cuda") for _ in range(2)]
    table = torch.tensor([[pages - 1, pages - 3, pages - 2]], dtype=torch.int32, device="cuda")
    for j in range(3):
        src, dst = int(small.table[0, j]), int(table[0, j])
        pool[0][dst], pool[1][dst] = small.k[src], small.v[src]
        scales[0][dst], scales[1][dst] = small.k_scales[src], small.v_scales[src]
    small.k, small.v, small.k_scales, small.v_scales, small.pages, small.table, small.table_dev = *pool, *scales, pages, table.cpu(), table
    assert pool[0].numel() > 1 << 32
    check(decode(small, q), *want, "far pages")


def test_decode_in_a_graph_and_on_another_stream():
    """Replays see what the buffers hold then; a call on a side stream."""
    c = Cache([300, 900, 0], heads=2, dim=128, page=64, dtype=INT8, block=16, seed=19)
    q = queries(3, 16, 128)
    d = cg.AttnDesc.make(16, 2, 128, num_seqs=3, total_q=3, max_kv=2000, scale=0.1)
    s = c.struct()
    ws, n = workspace(cg.codegemm_attn_decode_workspace_bytes(s, d))
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cg.codegemm_attn_decode(s, d, q, out, ws, n, side.cuda_stream)
    side.synchronize()
    check(out, *decode_exact(c, q, scale=0.1), "side stream")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        cg.codegemm_attn_decode(s, d, q, out, ws, n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    for k, lens in enumerate(([300, 900, 0], [17, 899, 0], [1, 64, 0], [300, 900, 0])):
        q.copy_(queries(3, 16, 128, seed=30 + k))
        c.lens_dev.copy_(torch.tensor(lens, dtype=torch.int32))
        c.lens = lens
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        check(got, *decode_exact(c, q, scale=0.1), f"replay {k}")
        cg.codegemm_attn_decode(s, d, q, out, ws, n, stream())
        torch.cuda.synchronize()
        assert torch.equal(got, out) and counters_are_clear()


# ---- packed prompts --------------------------------------------------------------------------------------------------------------

def packed(total_q, total_kv, Hq, Hk, D, seed=2):
    g = torch.Generator().manual_seed(seed)
    make = lambda n, h, s=1.0: (torch.randn(n, h, D, generator=g) * s).half().cuda()  # noqa: E731
    return make(total_q, Hq, 1.5), make(total_kv, Hk), make(total_kv, Hk)


@pytest.mark.parametrize("dim", [16, 48, 64, 80, 128, 192, 256])
@pytest.mark.parametrize("lens", [[1], [2, 1, 0, 31, 32, 33], [129], [64, 65, 63], [200, 7]])
def test_prompt_dims_and_lengths(dim, lens):
    q, k, v = packed(sum(lens), sum(lens), 4, 2, dim)
    check(prompt(q, k, v, lens, lens), *prompt_exact(q, k, v, lens, lens), f"D {dim} {lens}")


@pytest.mark.parametrize("heads,group", [(1, 1), (8, 1), (3, 5), (2, 8), (1, 17)])
def test_prompt_head_layouts(heads, group):
    q, k, v = packed(150, 150, heads * group, heads, 64)
    check(prompt(q, k, v, [50, 100], [50, 100]), *prompt_exact(q, k, v, [50, 100], [50, 100]), f"{heads} x {group}")


@pytest.mark.parametrize("group", [3, 7, 127, 128, 129, 1024])
def test_prompt_heads_that_share_a_tile(group):
    """Rows of a tile are query heads of some queries; where they do not divide evenly, a query's heads lie in two tiles or more."""
    new, total = [1, 3, 0, 9], [1, 80, 4, 70]
    if group < 100:
        new, total = [150, 3, 0, 61], [150, 80, 4, 300]
    q, k, v = packed(sum(new), sum(total), group, 1, 64)
    rows = set(range(0, sum(new), 9)) | {1, sum(new) - 1}
    for window, causal in ((0, True), (20, True), (0, False)):
        got = prompt(q, k, v, new, total, window=window, causal=causal)
        assert bool(got.isfinite().all())
        check(got[sorted(rows)], *prompt_exact(q, k, v, new, total, window=window, causal=causal, rows=rows), f"{group} heads, window {window}")


@pytest.mark.parametrize("new,total", [([5, 70], [300, 70]), ([1, 1, 1], [1, 64, 200]), ([33], [97]), ([40, 100], [10, 60]), ([20], [0]), ([0, 3], [50, 3]), ([130], [131])])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_lengths_of_queries_and_keys(new, total, causal):
    """Chunks behind a prefix, more queries than keys (the first see none), no keys at all."""
    q, k, v = packed(sum(new), max(1, sum(total)), 4, 2, 64)
    got = prompt(q, k, v, new, total, causal=causal)
    check(got, *prompt_exact(q, k, v, new, total, causal=causal), f"{new} of {total}")
    if causal and total[0] < new[0]:
        assert not bool(got[:new[0] - total[0]].any())


@pytest.mark.parametrize("window", [1, 2, 31, 32, 64, 65, 100, 1 << 30])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_window(window, causal):
    new, total = [150, 40, 10], [150, 260, 5]
    q, k, v = packed(sum(new), sum(total), 2, 1, 64)
    check(prompt(q, k, v, new, total, window=window, causal=causal), *prompt_exact(q, k, v, new, total, window=window, causal=causal), f"window {window}")


@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_prompt_what_a_query_does_not_see_does_not_reach_it(dim, bad):
    """A NaN or an infinity in a key or a value reaches the queries from its position on (and with a window, up to its end) and no other;
    nor do those of the sequences beside."""
    new = total = [90, 150, 40]
    q, k, v = packed(280, 280, 2, 1, dim)
    for window in (0, 20):
        kk, vv = k.clone(), v.clone()
        vv[90 + 70, 0, 3] = bad                    # of the second sequence, in the middle of a tile
        vv[90 + 71, 0, dim - 1] = bad
        kk[90 + 100, 0, 5] = bad
        kk[0], vv[0] = bad, bad                    # the first sequence: all of it
        got, (want, bound) = prompt(q, kk, vv, new, total, window=window), prompt_exact(q, kk, vv, new, total, window=window)
        clean, _ = prompt_exact(q, k, v, new, total, window=window)
        unaffected = list(range(90, 160)) + list(range(240, 280)) + (list(range(210, 240)) if window else [])
        assert bool(want[unaffected].isfinite().all()) and torch.equal(want[unaffected], clean[unaffected])
        check(got[unaffected], want[unaffected], bound[unaffected], f"unaffected rows, window {window}")
        fine = want.isfinite()
        assert bool((~got[~fine].isfinite()).all()), "a NaN that is seen has to be seen"
        # rows that see the bad values alone: their other dimensions are what they are without them
        want, bound = prompt_exact(q, k, vv.nan_to_num(0.0, 0.0, 0.0), new, total, window=window)
        rows = slice(90 + 72, 90 + (90 if window else 100))
        check(got[rows, :, 4:dim - 1], want[rows, :, 4:dim - 1], bound[rows, :, 4:dim - 1], f"other dimensions, window {window}")


def test_prompt_strides_and_scale():
    """q, k and v as columns of one fused projection's output, the result in rows of another width."""
    T, Hq, Hk, D = 77, 4, 2, 64
    g = torch.Generator().manual_seed(4)
    qkv = torch.randn(T, (Hq + 2 * Hk) * D + 8, generator=g).half().cuda()
    q, k, v = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D], qkv[:, (Hq + Hk) * D:(Hq + 2 * Hk) * D]
    out = torch.full((T, Hq * D + 24), 3.0, dtype=torch.float16, device="cuda")
    w = qkv.shape[1]
    for scale in (0.3, -0.1, 0.0):
        d = cg.AttnDesc.make(Hq, Hk, D, num_seqs=1, total_q=T, total_kv=T, max_kv=T, scale=scale, causal=True, q_stride=w, k_stride=w, v_stride=w, out_stride=Hq * D + 24)
        ws, n = workspace(cg.codegemm_attn_prompt_workspace_bytes(d))
        cg.codegemm_attn_prompt(d, q, k, v, starts([T]), None, out, ws, n, stream())
        want = prompt_exact(q.reshape(T, Hq, D), k.reshape(T, Hk, D), v.reshape(T, Hk, D), [T], [T], scale=scale)
        check(out[:, :Hq * D].reshape(T, Hq, D), *want, f"scale {scale}")
        assert bool((out[:, Hq * D:] == 3.0).all())


def test_prompt_peaked_scores():
    q, k, v = packed(260, 260, 2, 1, 128)
    k[200] *= 8
    check(prompt(q, k, v, [260], [260], scale=1.0), *prompt_exact(q, k, v, [260], [260], scale=1.0), "peaked")


@pytest.mark.parametrize("new,total", [([3000], [3000]), ([1024, 37, 700], [1024, 1500, 700]), ([16], [20000])])
def test_prompt_long(new, total):
    """Many tiles; a sample of the rows against 64 bits, and the same bits from call to call."""
    q, k, v = packed(sum(new), sum(total), 8, 1, 128)
    rows = set(range(0, sum(new), 173)) | {0, 1, sum(new) - 1, min(sum(new) - 1, 127), min(sum(new) - 1, 128)}
    got = prompt(q, k, v, new, total)
    check(got[sorted(rows)], *prompt_exact(q, k, v, new, total, rows=rows), f"{new} of {total}")
    assert torch.equal(got, prompt(q, k, v, new, total))


@pytest.mark.parametrize("dim", [64, 112, 128, 256])
@pytest.mark.parametrize("new,total", [([1], [700]), ([3, 0, 140], [900, 5, 1000]), ([17], [4000]), ([130, 20], [130, 2000])])
def test_prompt_few_queries_behind_long_prefixes(dim, new, total):
    """The keys of one tile of queries over several workgroups."""
    q, k, v = packed(sum(new), sum(total), 4, 2, dim)
    rows = set(range(0, sum(new), 13)) | {0, 2, sum(new) - 1}
    rows = {r for r in rows if r < sum(new)}
    for window, causal in ((0, True), (0, False), (500, True)):
        got = prompt(q, k, v, new, total, window=window, causal=causal)
        check(got[sorted(rows)], *prompt_exact(q, k, v, new, total, window=window, causal=causal, rows=rows), f"D {dim}, {new} of {total}, window {window}")
        assert torch.equal(got, prompt(q, k, v, new, total, window=window, causal=causal))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_prompt_what_a_query_does_not_see_in_any_part_of_the_keys(bad):
    """As above, where several workgroups share the keys: a bad value near the diagonal, and one at the lower end of the windows."""
    new, total, dim = [40], [1500], 128
    q, k, v = packed(40, 1500, 2, 1, dim)
    for window, at in ((0, 1480), (700, 1480), (700, 780)):
        vv = v.clone()
        vv[at, 0, 7] = bad
        got, (want, bound) = prompt(q, k, vv, new, total, window=window), prompt_exact(q, k, vv, new, total, window=window)
        seen = [i for i in range(40) if at <= 1460 + i and (not window or at > 1460 + i - window)]
        assert 0 < len(seen) < 40
        fine = want.isfinite()
        assert bool(fine[:, :, :7].all()) and int((~fine).sum()) == 2 * len(seen)
        check(got[fine], want[fine], bound[fine], f"window {window}, {at}")
        assert bool((~got[~fine].isfinite()).all())


@pytest.mark.parametrize("new", [[300, 1, 0, 129], [128] * 64, [5, 700, 256] + [0] * 61, [1] * 65, [400] + [3] * 70])
def test_prompt_order_of_sequences(new):
    """Up to as many sequences as a wavefront has lanes, and more: every tile is taken once."""
    q, k, v = packed(sum(new), sum(new), 16, 8, 64)
    rows = set(range(0, sum(new), 61)) | {0, sum(new) - 1}
    got = prompt(q, k, v, new, new)
    assert bool(got.isfinite().all())
    check(got[sorted(rows)], *prompt_exact(q, k, v, new, new, rows=rows), f"{len(new)} sequences")


# Thousands of tiles of queries and heads, whose keys no workgroups share; empty sequences stand for them here.
EMPTY = [0] * 4100


@pytest.mark.parametrize("dim", [16, 64, 80, 128, 256])
@pytest.mark.parametrize("new,total", [([1, 140], [1, 140]), ([129, 2], [300, 70]), ([40], [10]), ([200], [200])])
def test_prompt_with_thousands_of_tiles(dim, new, total):
    q, k, v = packed(sum(new), sum(total), 2, 1, dim)
    for window, causal in ((0, True), (0, False), (50, True)):
        got = prompt(q, k, v, new + EMPTY, total + EMPTY, window=window, causal=causal)
        check(got, *prompt_exact(q, k, v, new, total, window=window, causal=causal), f"D {dim}, {new} of {total}, window {window}")


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_prompt_what_a_query_does_not_see_with_thousands_of_tiles(dim, bad):
    q, k, v = packed(150, 400, 2, 1, dim)
    for window, at in ((0, 300), (0, 383), (100, 200)):
        vv = v.clone()
        vv[at, 0, 5] = bad
        got, (want, bound) = prompt(q, k, vv, [150] + EMPTY, [400] + EMPTY, window=window), prompt_exact(q, k, vv, [150], [400], window=window)
        seen = [i for i in range(150) if at <= 250 + i and (not window or at > 250 + i - window)]
        fine = want.isfinite()
        assert 0 < len(seen) < 150 and int((~fine).sum()) == 2 * len(seen)
        check(got[fine], want[fine], bound[fine], f"window {window}, {at}")
        assert bool((~got[~fine].isfinite()).all())


def test_prompt_many_sequences():
    """More sequences than a wavefront has lanes, some of them empty."""
    new = [(7 * i) % 5 for i in range(300)]
    q, k, v = packed(sum(new), sum(new), 2, 1, 64)
    check(prompt(q, k, v, new, new), *prompt_exact(q, k, v, new, new), "300 sequences")


def test_prompt_in_a_graph():
    new, total = [60, 100], [60, 200]
    q, k, v = packed(160, 260, 4, 2, 128)
    d = cg.AttnDesc.make(4, 2, 128, num_seqs=2, total_q=160, total_kv=260, max_kv=200, scale=0.1, causal=True)
    ws, n = workspace(cg.codegemm_attn_prompt_workspace_bytes(d))
    out, cu_q, cu_kv = torch.empty_like(q), starts(new), starts(total)
    cg.codegemm_attn_prompt(d, q, k, v, cu_q, cu_kv, out, ws, n, stream())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        cg.codegemm_attn_prompt(d, q, k, v, cu_q, cu_kv, out, ws, n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    for i, new in enumerate(([60, 100], [1, 159], [0, 160])):
        q.copy_(packed(160, 260, 4, 2, 128, seed=50 + i)[0])
        cu_q.copy_(starts(new))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        check(got, *prompt_exact(q, k, v, new, total, scale=0.1), f"replay {i}")
        cg.codegemm_attn_prompt(d, q, k, v, cu_q, cu_kv, out, ws, n, stream())
        torch.cuda.synchronize()
        assert torch.equal(got, out)

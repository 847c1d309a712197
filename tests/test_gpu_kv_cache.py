"""codegemm_kv_append and codegemm_kv_gather against their definitions: positions, norms and rotations, scales that grow, places that stay as they are."""
import pytest
import torch

pytestmark = pytest.mark.gpu

cg = pytest.importorskip("paper_2512_17970_amd")
from attention_util import QMAX, Cache, rope_table, rotated, starts  # noqa: E402
from gpu_util import Guarded, stream  # noqa: E402

FP16, INT8, FP8 = cg.binding.KV_FP16, cg.binding.KV_INT8, cg.binding.KV_FP8
EPS = 1e-5
# 32-bit rotation and norm against 64 bits: three roundings of products and sums of |a| + |b|, and for the norm a sum of D squares and a
# reciprocal root (some D / 2 + 8 roundings at most, half of them of the root's halved exponent)
F32 = 4 * 2.0 ** -24


def step(c, new, *, Hq=4, R=None, interleaved=False, norm=False, strides=False, in_place=False, seed=3, cu=True, size=1.0, positions=None, k_out=True):
    """One append; returns what went in (fp16) and came out."""
    g = torch.Generator().manual_seed(seed)
    T, H, D = sum(new), c.heads, c.dim
    R = D if R is None else R
    w = (Hq + 2 * H) * D + (16 if strides else 0)
    fused = (torch.randn(T, w, generator=g) * size).half().cuda()
    q, k, v = fused[:, :Hq * D], fused[:, Hq * D:(Hq + H) * D], fused[:, (Hq + H) * D:(Hq + 2 * H) * D]
    if not strides:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    ins = tuple(x.clone().reshape(T, -1, D) for x in (q, k, v))
    qn, kn = ((torch.randn(D, generator=g) * 0.2 + 1).half().cuda() for _ in range(2)) if norm else (None, None)
    rope = rope_table(positions or max(1, max(c.lens)), R) if R else None
    stride = w if strides else 0
    qg, kg = Guarded(T * Hq * D * 2), Guarded(T * H * D * 2)
    q_out = q if in_place else qg.view(torch.float16, (T, Hq * D)).fill_(float("nan"))
    ko = k if in_place else kg.view(torch.float16, (T, H * D)).fill_(float("nan"))
    if not k_out:
        ko = None
    d = cg.AppendDesc.make(T, Hq, rotary_dim=R, rope_positions=rope.shape[0] if R else 0, interleaved=interleaved, norm_eps=EPS, q_stride=stride, k_stride=stride, v_stride=stride,
                           q_out_stride=stride if in_place else 0, k_out_stride=stride if in_place else 0)
    cg.codegemm_kv_append(c.struct(), d, starts(new) if cu else None, q, k, v, qn, kn, rope, q_out, ko, stream())
    assert c.intact() and qg.intact() and kg.intact()
    at = torch.tensor([c.lens[i] - n + j for i, n in enumerate(new) for j in range(n)], device="cuda")
    want_q = rotated(ins[0], qn, at, rope, R, interleaved, EPS) if R or norm else ins[0].double()
    want_k = rotated(ins[1], kn, at, rope, R, interleaved, EPS) if R or norm else ins[1].double()
    loose = F32 * (12 + D) if norm else F32
    gone = at < 0
    want_q[gone], want_k[gone] = 0, 0
    for name, got, want in (("q_out", q_out, want_q), ("k_out", ko, want_k)):
        if got is None:
            continue
        size_ = want.abs().amax(-1, keepdim=True) * 2                  # |a| + |b| of a pair is at most that
        err = (got.reshape(want.shape).double() - want).abs()
        assert bool((err <= 2.0 ** -11 * want.abs() + loose * size_ + 2.0 ** -25).all()), f"{name}: {float(err.max())}"
    return want_k, ins[2].double(), loose


def check_cache(c, before, new, want_k, want_v, loose):
    """Every place of every pool: new tokens within half a step of what they are, earlier ones of a block that got a larger scale within half a step of
    what they were, all others bit for bit as before."""
    for pool, scales, old_pool, old_scales, want, values in ((c.k, c.k_scales, before[0], before[1], want_k, False), (c.v, c.v_scales, before[2], before[3], want_v, True)):
        expect, row = old_pool.clone(), 0
        slack = 0.0 if values else loose
        for i, n in enumerate(new):
            end, done = c.lens[i], set()
            begin = end - n
            for j in range(n):
                t = begin + j
                x, row = want[row], row + 1
                if t < 0 or c.page_of(i, t) is None:
                    continue
                got = c.place(pool, i, t, values)
                c.place(expect, i, t, values).copy_(got)
                if c.dtype == FP16:
                    assert bool(((got.double() - x).abs() <= 2.0 ** -11 * x.abs() + slack * 2 * x.abs().amax(-1, keepdim=True) + 2.0 ** -25).all())
                    continue
                b0 = t // c.block * c.block
                if b0 not in done:                                     # the block: its scale, and the tokens that were there
                    done.add(b0)
                    mine = [want[row - 1 + u - t] for u in range(max(b0, begin, 0), min(b0 + c.block, end))]
                    s = torch.stack(mine).abs().amax(0).amax(-1) / QMAX[c.dtype]
                    now, was = c.scale_of(scales, i, t).double(), c.scale_of(old_scales, i, t).double()
                    if b0 < begin:
                        s = torch.maximum(s, was)
                    assert bool(((now - s).abs() <= (2.0 ** -22 + 2 * slack) * s).all()), "scale"
                    for u in range(b0, max(begin, b0)):
                        prev, cur = c.place(old_pool, i, u, values).contiguous(), c.place(pool, i, u, values).contiguous()
                        c.place(expect, i, u, values).copy_(cur)
                        grown = now > was
                        assert torch.equal(prev[~grown], cur[~grown]), "earlier tokens under a scale that stayed"
                        exact = c.value(prev) * (was / now.clamp(min=1e-38))[:, None]
                        half = 0.5 if c.dtype == INT8 else exact.abs() * 2.0 ** -4 + 2.0 ** -10
                        assert bool(((c.value(cur) - exact).abs() <= half + 1e-4)[grown].all()), "earlier tokens in the larger scale"
                s = c.scale_of(scales, i, t).double()[:, None]
                half = 0.5 * s if c.dtype == INT8 else x.abs() * 2.0 ** -4 + s * 2.0 ** -10
                err = (c.value(got.contiguous()) * s - x).abs()
                assert bool((err <= half * (1 + 1e-4) + (slack + 2.0 ** -22) * 2 * x.abs().amax(-1, keepdim=True)).all()), f"new token {t} of {i}: {float((err / s.clamp(min=1e-30)).max())} steps"
        assert torch.equal(expect.view(torch.uint8), pool.view(torch.uint8)), "a place that is no token's was written"


def append(c, new, **kw):
    before = tuple(None if x is None else x.clone() for x in (c.k, c.k_scales, c.v, c.v_scales))
    out = step(c, new, **kw)
    check_cache(c, before, new, *out)


def grown(past, new):
    return [a + b for a, b in zip(past, new)]


TYPES = [(FP16, 1), (INT8, 1), (INT8, 4), (INT8, 16), (FP8, 1), (FP8, 8), (FP8, 16)]


@pytest.mark.parametrize("dtype,block", TYPES)
@pytest.mark.parametrize("dim", [16, 64, 80, 128, 256])
def test_append_types_and_dims(dtype, block, dim):
    past, new = [0, 0, 5, 16, 30, 7], [1, 40, 1, 17, 3, 0]
    append(Cache(grown(past, new), heads=2, dim=dim, dtype=dtype, block=block, seed=dim, filled=past), new, seed=dim + block)


@pytest.mark.parametrize("page,block", [(32, 32), (64, 2), (64, 64), (128, 32), (256, 256)])
@pytest.mark.parametrize("dtype", [INT8, FP8])
def test_append_blocks_and_pages(page, block, dtype):
    past, new = [0, 3, 100, 255, 250], [300, 1, 30, 2, 20]
    append(Cache(grown(past, new), heads=1, dim=64, page=page, dtype=dtype, block=block, seed=page, filled=past), new)


@pytest.mark.parametrize("page,block", [(32, 32), (64, 64), (128, 128), (256, 256)])
@pytest.mark.parametrize("dtype,dim", [(INT8, 128), (FP8, 64), (INT8, 256), (FP8, 16)])
def test_append_long_blocks_with_many_new_tokens(page, block, dtype, dim):
    """The 16-token groups of a block go round several teams of a workgroup."""
    past, new = [0, 37, 250], [301, 100, 17]
    append(Cache(grown(past, new), heads=1, dim=dim, page=page, dtype=dtype, block=block, seed=page, filled=past), new, norm=dim == 64)
    append(Cache(grown([5], [11]), heads=2, dim=dim, page=page, dtype=dtype, block=block, seed=page, filled=[5]), [11])


@pytest.mark.parametrize("size", [1e-3, 1.0, 30.0])
@pytest.mark.parametrize("dtype", [INT8, FP8])
def test_append_scales_grow_and_stay(size, dtype):
    """Token by token into blocks that hold smaller and larger ones."""
    past = [1, 5, 15, 17, 31]
    for round_ in range(3):
        new = [1] * 5
        append(Cache(grown(past, new), heads=2, dim=64, page=32, dtype=dtype, block=16, seed=round_, filled=past), new, cu=False, size=size, seed=round_, k_out=False)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [0, 16, 32, 64])
@pytest.mark.parametrize("norm", [False, True])
def test_append_rotations_and_norms(interleaved, R, norm):
    past, new = [0, 9, 200], [20, 1, 5]
    append(Cache(grown(past, new), heads=3, dim=64, dtype=INT8, block=4, seed=R, filled=past), new, R=R, interleaved=interleaved, norm=norm)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dim", [48, 128])
def test_append_from_a_fused_projection(in_place, dim):
    past, new = [0, 40], [33, 2]
    append(Cache(grown(past, new), heads=2, dim=dim, dtype=FP8, block=16, seed=1, filled=past), new, strides=True, in_place=in_place, norm=True)


def test_append_many_tokens_and_heads():
    """Enough tokens that a workgroup takes all heads of one, and more sequences than a wavefront has lanes."""
    new = [(11 * i) % 29 for i in range(90)]
    past = [(5 * i) % 23 for i in range(90)]
    assert sum(new) >= 1024
    append(Cache(grown(past, new), heads=1, dim=64, dtype=INT8, block=16, seed=2, filled=past), new, Hq=40)


def test_append_rows_without_a_place():
    """Idle slots (length 0), lengths shorter than the new tokens, pages that are missing: nothing is written, q_out and k_out are zero at negative positions."""
    for dtype, block in ((FP16, 1), (INT8, 4), (INT8, 16)):
        c = Cache([0, 3, 40], heads=1, dim=64, dtype=dtype, block=block, seed=4, filled=[0, 0, 20])
        c.table[2, 1] = -1                                             # positions 16..31
        c.table[2, 2] = c.pages + 5                                    # 32..
        c.table_dev.copy_(c.table)
        append(c, [1, 5, 20])


def test_append_positions_past_the_table_take_its_last_row():
    past, new = [60], [10]
    append(Cache(grown(past, new), heads=1, dim=64, dtype=FP16, seed=4, filled=past), new, positions=63)


@pytest.mark.parametrize("dtype,block", [(FP16, 1), (INT8, 1), (INT8, 16)])
def test_append_lengths_beyond_the_page_table(dtype, block):
    """Up to the largest there are: no place in the cache, q_out and k_out turned by the rope table's last row."""
    c = Cache([64, 64, 64], heads=1, dim=64, dtype=dtype, block=block, seed=4)
    c.lens_dev.copy_(torch.tensor([2 ** 31 - 1, 2 ** 31 - 20, 64 + 40], dtype=torch.int32))
    before = [x.clone() for x in (c.k, c.v)]
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(120, 64, generator=g).half().cuda() for _ in range(3))
    rope = rope_table(64, 64)
    q_out, k_out = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    d = cg.AppendDesc.make(120, 1, rotary_dim=64, rope_positions=64)
    cg.codegemm_kv_append(c.struct(), d, starts([40, 40, 40]), q, k, v, None, None, rope, q_out, k_out, stream())
    torch.cuda.synchronize()
    assert c.intact() and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, (c.k, c.v)))
    at = torch.full((120,), 63, device="cuda")
    for got, x in ((q_out, q), (k_out, k)):
        want = rotated(x[:, None], None, at, rope, 64, False, EPS)[:, 0]
        assert bool(((got.double() - want).abs() <= 2.0 ** -11 * want.abs() + F32 * 2 * want.abs().amax() + 2.0 ** -25).all())


def test_append_nan_and_infinity():
    """A block that gets one reads as NaN, alone; it starts afresh with its first token."""
    for dtype in (INT8, FP8):
        for bad in (float("nan"), float("inf"), float("-inf")):
            c = Cache([40], heads=2, dim=64, dtype=dtype, block=4, seed=6, filled=[35])
            g = torch.Generator().manual_seed(1)
            q, k, v = ((torch.randn(5, h * 64, generator=g)).half().cuda() for h in (2, 2, 2))
            k[1, 3] = bad                                              # position 36 of head 0: block 36..39
            v[4, 64] = bad                                             # position 39 of head 1
            d = cg.AppendDesc.make(5, 2)
            q_out, k_out = torch.empty_like(q), torch.empty_like(k)
            cg.codegemm_kv_append(c.struct(), d, starts([5]), q, k, v, None, None, None, q_out, k_out, stream())
            assert c.intact()
            keys = torch.stack([c.read(0, t, False) for t in range(40)])
            values = torch.stack([c.read(0, t, True) for t in range(40)])
            assert bool(keys[36:, 0].isnan().all()) and bool(keys[:36].isfinite().all()) and bool(keys[:, 1].isfinite().all())
            assert bool(values[36:, 1].isnan().all()) and bool(values[:36].isfinite().all()) and bool(values[:, 0].isfinite().all())
            # one more token stays in the NaN block's shadow only where the block is not new
            k[:], v[:] = 1.0, 1.0
            c.lens_dev.fill_(37)
            cg.codegemm_kv_append(c.struct(), cg.AppendDesc.make(1, 2), None, q, k, v, None, None, None, q_out, k_out, stream())
            torch.cuda.synchronize()
            for values in (False, True):                               # the largest code times a scale that is rounded to 24 bits
                assert bool(((c.read(0, 36, values) - 1.0).abs() <= 2.0 ** -24).all())


def test_append_zeros_and_tiny_values():
    for dtype in (INT8, FP8):
        c = Cache([2], heads=1, dim=16, dtype=dtype, block=1, seed=6, filled=[0])
        z = torch.zeros(2, 16, dtype=torch.float16, device="cuda")
        z[1, 5] = 6e-8                                                 # the least subnormal
        cg.codegemm_kv_append(c.struct(), cg.AppendDesc.make(2, 0), starts([2]), None, z, z, None, None, None, None, None, stream())
        for values in (False, True):
            assert bool((c.read(0, 0, values) == 0).all())
            assert torch.allclose(c.read(0, 1, values)[0], z[1].double(), rtol=1e-3, atol=0)


def test_append_then_append_again_gives_the_same():
    past, new = [5, 0], [30, 3]
    c = Cache(grown(past, new), heads=2, dim=64, dtype=INT8, block=16, seed=8, filled=past)
    step(c, new)
    first = [x.clone() for x in (c.k, c.v, c.k_scales, c.v_scales)]
    step(c, new)
    for a, b in zip(first, (c.k, c.v, c.k_scales, c.v_scales)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("dtype,block", TYPES)
@pytest.mark.parametrize("dim", [16, 80, 128, 256])
def test_gather(dtype, block, dim):
    lens, first, rows = [50, 0, 17, 100, 20], [0, 0, 3, 31, -5], [50, 4, 14, 69, 30]
    c = Cache(lens, heads=3, dim=dim, page=32, dtype=dtype, block=block, seed=dim)
    c.table[3, 2] = -7                                                 # positions 64..95
    c.table_dev.copy_(c.table)
    T = sum(rows)
    gk, gv = Guarded(T * 3 * dim * 2), Guarded(T * 3 * dim * 2)
    k, v = (g.view(torch.float16, (T, 3, dim)).fill_(float("nan")) for g in (gk, gv))
    f = torch.tensor(first, dtype=torch.int32, device="cuda")
    cg.codegemm_kv_gather(c.struct(), T, starts(rows), f, k, v, stream())
    assert c.intact() and gk.intact() and gv.intact()
    row = 0
    for i, n in enumerate(rows):
        for j in range(n):
            t = first[i] + j
            for got, values in ((k, False), (v, True)):
                want = c.read(i, t, values) if 0 <= t < lens[i] else None
                want = torch.zeros(3, dim, dtype=torch.float64, device="cuda") if want is None else want
                # one product of 8 by 24 bits in 32 bits and one rounding to fp16
                assert bool(((got[row].double() - want).abs() <= (2.0 ** -11 + 2.0 ** -23) * want.abs() + 2.0 ** -25).all()), (i, t, values)
            row += 1
    one = torch.full_like(k, float("nan"))
    cg.codegemm_kv_gather(c.struct(), T, starts(rows), f, None, one, stream())
    assert torch.equal(one, v)
    cg.codegemm_kv_gather(c.struct(), T, starts(rows), f, one, None, stream())
    assert torch.equal(one, k)


def test_append_and_gather_in_a_graph():
    """A decoding step captured once: the lengths grow on the device between replays."""
    c = Cache([64, 64], heads=2, dim=64, page=32, dtype=INT8, block=16, seed=3, filled=[20, 31])
    g = torch.Generator().manual_seed(9)
    q, k, v = (torch.randn(2, n * 64, generator=g).half().cuda() for n in (4, 2, 2))
    rope = rope_table(64, 64)
    q_out = torch.empty_like(q)
    s, d = c.struct(), cg.AppendDesc.make(2, 4, rotary_dim=64, rope_positions=64)
    keys, values = torch.empty(2, 2, 64, dtype=torch.float16, device="cuda"), torch.empty(2, 2, 64, dtype=torch.float16, device="cuda")
    last, cu = torch.tensor([20, 31], dtype=torch.int32, device="cuda"), starts([1, 1])
    c.lens_dev.copy_(last + 1)

    def issue(stream_):
        cg.codegemm_kv_append(s, d, None, q, k, v, None, None, rope, q_out, None, stream_)
        cg.codegemm_kv_gather(s, 2, cu, last, keys, values, stream_)
        c.lens_dev.add_(1)
        last.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        issue(torch.cuda.current_stream().cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    for k_ in range(6):
        k.copy_(torch.randn(2, 128, generator=g).half())
        v.copy_(torch.randn(2, 128, generator=g).half())
        at = torch.tensor([20 + k_, 31 + k_], device="cuda")
        graph.replay()
        torch.cuda.synchronize()
        want = rotated(k.reshape(2, 2, 64), None, at, rope, 64, False, EPS)
        for got, exact, scales in ((keys, want, c.k_scales), (values, v.reshape(2, 2, 64).double(), c.v_scales)):
            # half a step, and the rounding of what is read to fp16
            assert bool(((got.double() - exact).abs() <= 0.51 * float(scales.nan_to_num().max()) + 2.0 ** -11 * exact.abs()).all())

"""The cache in 4 bits: codegemm_kv_append, codegemm_kv_append_shifted, codegemm_kv_gather and codegemm_attn_decode against their definitions in 64 bits, from the
documented layout."""
import pytest
import torch

pytestmark = pytest.mark.gpu

cg = pytest.importorskip("paper_2512_17970_amd")
from attention_util import attention, check, counters_are_clear, rope_table, rotated, starts, workspace  # noqa: E402
from gpu_util import Guarded, stream  # noqa: E402

from four_bits_util import Cache4  # noqa: E402

EPS = 1e-5
F32 = 4 * 2.0 ** -24          # rotation in 32 bits: three roundings of products and sums of |a| + |b|


def step(c, new, *, Hq=4, R=None, interleaved=False, norm=False, strides=False, in_place=False, seed=3, cu=True, size=1.0, positions=None, k_out=True, shift=None, spoil=()):
    """One append; returns what the cache should stand for: keys and values in 64 bits before they are coded, and what the keys' 32 bits may be off by."""
    g = torch.Generator().manual_seed(seed)
    T, H, D = sum(new), c.heads, c.dim
    R = D if R is None else R
    w = (Hq + 2 * H) * D + (16 if strides else 0)
    fused = (torch.randn(T, w, generator=g) * size).half().cuda()
    for row, col, x in spoil:
        fused[row, col] = x
    q, k, v = fused[:, :Hq * D], fused[:, Hq * D:(Hq + H) * D], fused[:, (Hq + H) * D:(Hq + 2 * H) * D]
    if not strides:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    ins = tuple(x.clone().reshape(T, -1, D) for x in (q, k, v))
    qn, kn = ((torch.randn(D, generator=g) * 0.2 + 1).half().cuda() for _ in range(2)) if norm else (None, None)
    rope = rope_table(positions or max(1, max(c.lens)) + max(shift or [0]), R) if R else None
    stride = w if strides else 0
    qg, kg = Guarded(T * Hq * D * 2), Guarded(T * H * D * 2)
    q_out = q if in_place else qg.view(torch.float16, (T, Hq * D)).fill_(float("nan"))
    ko = k if in_place else kg.view(torch.float16, (T, H * D)).fill_(float("nan"))
    ko = ko if k_out else None
    d = cg.AppendDesc.make(T, Hq, rotary_dim=R, rope_positions=rope.shape[0] if R else 0, interleaved=interleaved, norm_eps=EPS, q_stride=stride, k_stride=stride, v_stride=stride,
                           q_out_stride=stride if in_place else 0, k_out_stride=stride if in_place else 0)
    rest = (q, k, v, qn, kn, rope, q_out, ko, stream())
    if shift is None:
        cg.codegemm_kv_append(c.struct(), d, starts(new) if cu else None, *rest)
    else:
        cg.codegemm_kv_append_shifted(c.struct(), d, starts(new) if cu else None, torch.tensor(shift, dtype=torch.int32, device="cuda"), *rest)
    assert c.intact() and qg.intact() and kg.intact()
    place = torch.tensor([c.lens[i] - n + j for i, n in enumerate(new) for j in range(n)], device="cuda")
    at = place + torch.tensor([(shift or [0] * len(new))[i] for i, n in enumerate(new) for _ in range(n)], device="cuda")
    want_q = rotated(ins[0], qn, at, rope, R, interleaved, EPS) if R or norm else ins[0].double()
    want_k = rotated(ins[1], kn, at, rope, R, interleaved, EPS) if R or norm else ins[1].double()
    loose = F32 * (12 + D) if norm else F32
    if spoil:
        return want_k, ins[2].double(), loose
    gone = place < 0
    want_q[gone], want_k[gone] = 0, 0
    for name, got, want in (("q_out", q_out, want_q), ("k_out", ko, want_k)):
        if got is not None:
            err = (got.reshape(want.shape).double() - want).abs()
            assert bool((err <= 2.0 ** -11 * want.abs() + loose * want.abs().amax(-1, keepdim=True) * 2 + 2.0 ** -25).all()), f"{name}: {float(err.max())}"
    return want_k, ins[2].double(), loose


def check_cache(c, before, new, want_k, want_v, loose):
    """Every place of every pool: scales and offsets within a rounding of what the definition gives, the codes such that the value is within half a step (and
    what scale and offset are rounded by); all other places bit for bit as they were."""
    for values, want in ((False, want_k), (True, want_v)):
        expect, expect_s = c.copy_of(before, values)
        slack, row = 0.0 if values else loose, 0
        for i, n in enumerate(new):
            for j in range(n):
                t = c.lens[i] - n + j
                x, row = want[row], row + 1
                if t < 0 or c.page_of(i, t) is None:
                    continue
                code, s, o = (y.double() for y in c.raw(i, t, values))
                c.accept(expect, expect_s, i, t, values)
                err_x = 2 * slack * x.abs().amax(-1, keepdim=True)                              # of x itself
                for r in range(c.runs):
                    mine = slice(r * c.block, min(c.dim, (r + 1) * c.block))
                    lo, hi = x[:, mine].amin(-1), x[:, mine].amax(-1)
                    step_ = (hi - lo) * (1 - 2.0 ** -11) / 15
                    size = err_x[:, 0] + 2.0 ** -23 * (lo.abs() + hi.abs())
                    assert bool(((s[:, r] - step_).abs() <= 2.0 ** -11 * step_ + size + 2.0 ** -25).all()), "scale"
                    assert bool(((o[:, r] - (lo - 16 * s[:, r])).abs() <= 2.0 ** -11 * (lo - 16 * s[:, r]).abs() + size + 2.0 ** -25).all()), "offset"
                    # the nearest of the 16 values (offset + 16 .. 31 scales): within half a step where x lies among them, and what lies beyond is off by the
                    # roundings of scale and offset: 15 (2^-10 + 2^-24 of a scale's own rounding) scales and 2^-11 of the offset
                    value = (code[:, mine] + 16) * s[:, r:r + 1] + o[:, r:r + 1]
                    end = 15 * 2.0 ** -10 * s[:, r] + 2.0 ** -11 * o[:, r].abs() + 15 * 2.0 ** -25 + 2.0 ** -24
                    bound = 0.5 * s[:, r] * (1 + 2.0 ** -18) + end
                    assert bool(((value - x[:, mine]).abs() <= bound[:, None] + err_x + 2.0 ** -22 * (x[:, mine].abs() + o[:, r:r + 1].abs())).all()), f"token {t} of {i}"
        assert c.same(expect, expect_s, values), "a place that is no token's was written"


def append(c, new, **kw):
    before = c.snapshot()
    check_cache(c, before, new, *step(c, new, **kw))


def grown(past, new):
    return [a + b for a, b in zip(past, new)]


@pytest.mark.parametrize("dim,block", [(32, 32), (64, 32), (64, 64), (96, 32), (96, 64), (128, 32), (128, 64), (128, 128), (160, 32), (224, 128), (256, 32), (256, 256), (64, 256)])
def test_append_dims_and_runs(dim, block):
    past, new = [0, 0, 5, 16, 30, 7], [1, 40, 1, 17, 3, 0]
    append(Cache4(grown(past, new), heads=2, dim=dim, block=block, seed=dim, filled=past), new, seed=dim + block)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_append_pages(page):
    past, new = [0, 3, 100, 255, 250], [300, 1, 30, 2, 20]
    append(Cache4(grown(past, new), heads=1, dim=64, page=page, seed=page, filled=past), new)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [0, 16, 32, 48, 96])
@pytest.mark.parametrize("norm", [False, True])
def test_append_rotations_and_norms(interleaved, R, norm):
    past, new = [0, 9, 200], [20, 1, 5]
    append(Cache4(grown(past, new), heads=3, dim=96, seed=R, filled=past), new, R=R, interleaved=interleaved, norm=norm)


@pytest.mark.parametrize("dim", [64, 128])
def test_append_strides_and_in_place(dim):
    past, new = [0, 31, 64], [33, 1, 15]
    for kw in (dict(strides=True), dict(strides=True, in_place=True), dict(in_place=True), dict(k_out=False)):
        append(Cache4(grown(past, new), heads=2, dim=dim, page=32, filled=past), new, **kw)


@pytest.mark.parametrize("size", [1e-6, 1e-3, 30.0, 5000.0])
def test_append_sizes(size):
    """Small values, whose scales are subnormal, and large ones (5000 times a normal deviate is seldom beyond 20000)."""
    c = Cache4([20, 1], heads=2, dim=64, filled=[0, 0])
    append(c, [20, 1], size=size, R=0, seed=5)


def test_append_one_value_and_values_beyond_the_range():
    c = Cache4([3], heads=1, dim=64, filled=[0])
    k = torch.full((3, 64), 1.5).half()
    k[1] = -60000.0
    k[2, :32], k[2, 32:] = 65504.0, torch.linspace(-60000, 60000, 32).half()
    k = k.cuda()
    d = cg.AppendDesc.make(3, 0)
    cg.codegemm_kv_append(c.struct(), d, starts([3]), None, k, k, None, None, None, None, None, stream())
    assert c.intact()
    for values in (False, True):
        got = [c.read(0, t, values)[0] for t in range(3)]
        assert bool((got[0] == 1.5).all())
        assert bool(((got[1] + 20000).abs() <= 16).all()) and bool(((got[2][:32] - 20000).abs() <= 16).all())        # the offset's half unit in fp16
        held = k[2, 32:].double().clamp(-20000, 20000)
        assert bool(((got[2][32:] - held).abs() <= 0.5 * 40000 / 15 + 100).all())


def test_append_runs_with_nan_and_infinity():
    """Such a run reads as NaN, its neighbours and other tokens as they are."""
    for x in (float("nan"), float("inf"), float("-inf")):
        for values in (False, True):
            c = Cache4([20], heads=1, dim=64, filled=[0])
            col = 64 + (64 if values else 0) + 40                     # one head of q: dimension 40, in the second run
            want_k, want_v, _ = step(c, [20], Hq=1, R=0, spoil=[(7, col, x)])
            for t in range(20):
                got = c.read(0, t, values)[0]
                assert bool(got[32:].isnan().all()) == (t == 7) and bool(got[:32].isfinite().all()) and bool((t == 7) | got[32:].isfinite().all())


def test_idle_slots_absent_pages_and_lengths_beyond_the_table():
    c = Cache4([5, 0, 40, 33], heads=2, dim=64, filled=[4, 0, 39, 32])
    c.table[2, 2] = c.pages + 5
    c.table[3, 2] = -1
    c.table_dev.copy_(c.table.cuda())
    append(c, [1, 1, 1, 1], cu=False)
    c = Cache4([5, 70], heads=2, dim=64, filled=[4, 0], max_pages=4)
    append(c, [1, 70], k_out=True)


@pytest.mark.parametrize("shift", [[0, 0, 0], [7, 100, 1], [3, 0, 1 << 29]])
def test_append_shifted(shift):
    past, new = [0, 9, 30], [20, 1, 5]
    c = Cache4(grown(past, new), heads=2, dim=64, filled=past)
    append(c, new, shift=shift, positions=150)


def test_append_shifted_below_the_table_and_other_types():
    """Positions below 0 take the first row.  The other types' keys turn alike: k_out says so."""
    for dtype in (cg.KV_FP16, cg.KV_INT8):
        from attention_util import Cache
        past, new, shift = [0, 9], [20, 1], [50, -40]
        c = Cache(grown(past, new), heads=2, dim=64, dtype=dtype, block=16 if dtype else 1, filled=past)
        step(c, new, shift=shift, positions=60)
    c = Cache4([10], heads=1, dim=64, filled=[0])
    append(c, [10], shift=[-3])


def gather(c, lens, first, out=True):
    rows, H, D = sum(lens), c.heads, c.dim
    gk, gv = Guarded(rows * H * D * 2), Guarded(rows * H * D * 2)
    k, v = gk.view(torch.float16, (rows, H, D)).fill_(float("nan")), gv.view(torch.float16, (rows, H, D)).fill_(float("nan"))
    cg.codegemm_kv_gather(c.struct(), rows, starts(lens), None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda"), k, v, stream())
    assert gk.intact() and gv.intact() and c.intact()
    row = 0
    for i, n in enumerate(lens):
        for j in range(n):
            t = j + (first[i] if first else 0)
            for got, values in ((k, False), (v, True)):
                want = c.read(i, t, values) if 0 <= t < c.lens[i] else None
                want = torch.zeros(H, D, dtype=torch.float64, device="cuda") if want is None else want
                assert torch.equal(got[row].double(), want), (i, t, values)      # a cached value is a number in fp16
            row += 1


@pytest.mark.parametrize("dim,block,page", [(32, 32, 16), (64, 32, 32), (96, 64, 16), (128, 32, 64), (128, 128, 256), (256, 64, 16), (160, 256, 128)])
def test_gather(dim, block, page):
    c = Cache4([1, 37, 0, 100, 15], heads=2, dim=dim, block=block, page=page, seed=dim)
    c.table[3, 0] = -7
    c.table_dev.copy_(c.table.cuda())
    gather(c, [1, 37, 3, 100, 16], None)
    gather(c, [2, 20, 0, 31, 40], [0, 9, 0, 70, -20])


def decode(c, q, *, window=0, scale=None, max_kv=None, q_stride=0, out_stride=0):
    B, Hq, D = q.shape
    d = cg.AttnDesc.make(Hq, c.heads, D, num_seqs=B, total_q=B, max_kv=max_kv or max(1, max(c.lens)), scale=D ** -0.5 if scale is None else scale, window=window,
                         q_stride=q_stride, out_stride=out_stride)
    s = c.struct()
    ws, n = workspace(cg.codegemm_attn_decode_workspace_bytes(s, d))
    g = Guarded(B * Hq * D * 2)
    out = g.view(torch.float16, (B, Hq, D)).fill_(float("nan"))
    cg.codegemm_attn_decode(s, d, q, out, ws, n, stream())
    assert g.intact() and c.intact() and counters_are_clear()
    return out


def decode_exact(c, q, window=0, scale=None):
    out, bound = [], []
    for i, n in enumerate(c.lens):
        k, v, seen = c.sequence(i, max(0, n - window) if window else 0, n)
        o, b = attention(q[i], k, v, seen, c.dim ** -0.5 if scale is None else scale)
        out.append(o)
        bound.append(b)
    return torch.stack(out), torch.stack(bound)


def queries(B, Hq, D, seed=1, size=1.5):
    return (torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(seed)) * size).half().cuda()


@pytest.mark.parametrize("dim,block", [(32, 32), (64, 32), (64, 64), (96, 32), (96, 64), (128, 32), (128, 64), (128, 128), (160, 32), (192, 128), (256, 32), (256, 256)])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 8), (3, 5), (1, 17)])
def test_decode_dims_and_heads(dim, block, heads, group):
    c = Cache4([1, 37, 0, 100, 15, 64], heads=heads, dim=dim, block=block, page=16, seed=dim)
    q = queries(6, heads * group, dim)
    check(decode(c, q), *decode_exact(c, q), f"{dim} {block}")


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window", [0, 1, 33, 500])
def test_decode_pages_and_windows(page, window):
    c = Cache4([700, 3, 257, 0, 31, 1000], heads=2, dim=64, page=page, seed=page)
    q = queries(6, 8, 64)
    check(decode(c, q, window=window), *decode_exact(c, q, window), f"{page} {window}")


def test_decode_without_some_pages():
    c = Cache4([300, 90, 16, 40], heads=2, dim=128, page=16, seed=4)
    c.table[0, 3:7] = -1
    c.table[0, 18] = c.pages
    c.table[1, :] = -5
    c.table[3, 2] = 1 << 30
    c.table_dev.copy_(c.table.cuda())
    q = queries(4, 16, 128)
    got = decode(c, q)
    check(got, *decode_exact(c, q), "absent pages")
    assert bool((got[1] == 0).all())


def test_decode_lengths_beyond_the_table_and_below_zero():
    c = Cache4([40, -3, 64], heads=1, dim=64, page=16, max_pages=4)
    c.lens_dev.copy_(torch.tensor([1000, -3, 1 << 30], dtype=torch.int32))
    q = queries(3, 4, 64)
    got = decode(c, q)
    c.lens = [48, 0, 64]                                                # places 40 to 47 hold what the cache was filled with: not looked at here
    want, bound = decode_exact(c, q)
    check(got[1:], want[1:], bound[1:], "lengths")


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0, 1e30])
def test_decode_scales(scale):
    c = Cache4([77, 200], heads=2, dim=64, seed=9)
    q = queries(2, 4, 64)
    want, bound = decode_exact(c, q, scale=min(scale, 1e25))
    if abs(scale) < 1e3:
        check(decode(c, q, scale=scale), want, bound, f"{scale}")
    else:
        got = decode(c, q, scale=scale).double()                        # all weight goes to one key
        assert bool((got - want).abs().max() <= 2.0 ** -10 * want.abs().max())


@pytest.mark.parametrize("heads,group,dim", [(8, 8, 128), (2, 4, 64), (1, 1, 256)])
def test_decode_long(heads, group, dim):
    """In pieces, joined; the same bits again; more sequences than a wavefront looks at in one go."""
    c = Cache4([9000, 1, 4100], heads=heads, dim=dim, page=64, seed=2, quick=True)
    q = queries(3, heads * group, dim)
    got = decode(c, q)
    check(got, *decode_exact(c, q), "long")
    assert torch.equal(decode(c, q), got) and torch.equal(decode(c, q, max_kv=1), decode(c, q, max_kv=1))
    check(decode(c, q, max_kv=1), *decode_exact(c, q), "longer than the host knows")


def test_decode_many_sequences():
    lens = [(37 * i) % 90 for i in range(300)]
    c = Cache4(lens, heads=2, dim=64, page=16, seed=3, quick=True)
    q = queries(300, 4, 64)
    check(decode(c, q), *decode_exact(c, q), "many")


def test_decode_strides_and_another_stream():
    c = Cache4([100, 257], heads=2, dim=128, page=32, seed=6)
    q = queries(2, 8, 128)
    wide = torch.zeros(2, 8 * 128 + 64, dtype=torch.float16, device="cuda")
    wide[:, :1024] = q.view(2, -1)
    want = decode(c, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s, d = c.struct(), cg.AttnDesc.make(8, 2, 128, num_seqs=2, total_q=2, max_kv=257, scale=128 ** -0.5, q_stride=wide.shape[1], out_stride=1024 + 8)
        ws = torch.zeros(cg.codegemm_attn_decode_workspace_bytes(s, d), dtype=torch.uint8, device="cuda")
        out = torch.full((2, 1032), 7.0, dtype=torch.float16, device="cuda")
        cg.codegemm_attn_decode(s, d, wide, out, ws, ws.numel(), stream())
    torch.cuda.synchronize()
    assert torch.equal(out[:, :1024].reshape(2, 8, 128), want) and bool((out[:, 1024:] == 7).all())


def test_a_step_in_a_graph():
    """Append and attention in a graph, lengths on the device, eager work between replays: the same bits as eager calls."""
    H, D, B = 2, 64, 3
    lens = [20, 1, 47]
    a, b = (Cache4(lens, heads=H, dim=D, page=16, seed=8, max_pages=8) for _ in range(2))
    for c in (a, b):                                                    # pages for what is to come
        for i in range(B):
            for j in range(8):
                c.table[i, j] = i * 8 + j if c.table[i, j] < 0 else c.table[i, j]
        c.remap(torch.arange(B * 8).view(B, 8))
    g = torch.Generator().manual_seed(1)
    xs = [(torch.randn(B, (4 + 2 * H) * D, generator=g)).half().cuda() for _ in range(6)]
    rope = rope_table(200, D)

    def step_of(c, x, q_out, out, ws):
        d = cg.AppendDesc.make(B, 4, rotary_dim=D, rope_positions=200, q_stride=x.shape[1], k_stride=x.shape[1], v_stride=x.shape[1])
        t = cg.AttnDesc.make(4, H, D, num_seqs=B, total_q=B, max_kv=128, scale=D ** -0.5)
        c.lens_dev += 1
        s = c.struct()
        cg.codegemm_kv_append(s, d, None, x[:, :4 * D], x[:, 4 * D:(4 + H) * D], x[:, (4 + H) * D:], None, None, rope, q_out, None, stream())
        cg.codegemm_attn_decode(s, t, q_out, out, ws, ws.numel(), stream())

    bufs = [(torch.empty(B, 4, D, dtype=torch.float16, device="cuda"), torch.empty(B, 4, D, dtype=torch.float16, device="cuda"),
             torch.zeros(8 << 20, dtype=torch.uint8, device="cuda")) for _ in range(2)]
    x = xs[0].clone()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    step_of(b, x, *bufs[1])
    b.lens_dev -= 1
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step_of(b, x, *bufs[1])
    for x_now in xs:
        step_of(a, x_now, *bufs[0])
        x.copy_(x_now)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bufs[0][1], bufs[1][1]) and torch.equal(bufs[0][0], bufs[1][0])
    assert torch.equal(a.lens_dev, b.lens_dev)

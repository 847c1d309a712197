"""Corners of the cache and of attention: blocks whose scale is a NaN, keys and values in rows of different widths, gathers of 2^32 threads and more."""
import pytest
import torch

pytestmark = pytest.mark.gpu

cg = pytest.importorskip("paper_2512_17970_amd")
from attention_util import Cache, check, decode, decode_exact, prompt_exact, starts, workspace  # noqa: E402
from gpu_util import stream  # noqa: E402

FP16, INT8, FP8 = cg.binding.KV_FP16, cg.binding.KV_INT8, cg.binding.KV_FP8


def queries(B, Hq, D):
    return (torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(1)) * 1.5).half().cuda()


@pytest.mark.parametrize("lens", [[70, 200, 33], [900, 3000, 5]])
@pytest.mark.parametrize("dtype,block,dim", [(INT8, 1, 64), (INT8, 4, 128), (INT8, 16, 128), (FP8, 64, 64), (FP8, 16, 256)])
@pytest.mark.parametrize("of", ["k_scales", "v_scales"])
def test_decode_over_a_block_whose_scale_is_nan(lens, dtype, block, dim, of):
    """All of its tokens read as NaN, so every query that sees it gets NaN, and no other: not the other head's, not those whose window lies behind it."""
    c = Cache(lens, heads=2, dim=dim, page=64, dtype=dtype, block=block, seed=3)
    q, at = queries(3, 4, dim), 20
    want, bound = decode_exact(c, q)
    near = decode_exact(c, q, window=5)
    c.scale_of(getattr(c, of), 1, at)[0] = float("nan")                    # sequence 1, key head 0: query heads 0 and 1
    got = decode(c, q)
    assert bool(got[1, :2].isnan().all())
    got[1, :2], want[1, :2] = 0, 0
    check(got, want, bound, "without the block")
    check(decode(c, q, window=5), *near, "behind the block")


@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("extra", [(0, 8, 264), (16, 72, 0), (8, 1024, 40)])
def test_prompt_rows_of_different_widths(dim, extra):
    """Queries, keys and values in rows of their own widths; masked and whole tiles, keys shared by workgroups."""
    new, total, Hq, Hk = [5, 140], [300, 140], 4, 2
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(sum(n), h * dim + e, generator=g).half().cuda() for n, h, e in ((new, Hq, extra[0]), (total, Hk, extra[1]), (total, Hk, extra[2])))
    out = torch.full((sum(new), Hq * dim), float("nan"), dtype=torch.float16, device="cuda")
    dense = [x[:, :h * dim].reshape(x.shape[0], h, dim) for x, h in ((q, Hq), (k, Hk), (v, Hk))]
    for window in (0, 50):
        d = cg.AttnDesc.make(Hq, Hk, dim, num_seqs=2, total_q=sum(new), total_kv=sum(total), max_kv=300, scale=dim ** -0.5, window=window, causal=True,
                             q_stride=q.shape[1], k_stride=k.shape[1], v_stride=v.shape[1])
        ws, n = workspace(cg.codegemm_attn_prompt_workspace_bytes(d))
        cg.codegemm_attn_prompt(d, q, k, v, starts(new), starts(total), out, ws, n, stream())
        check(out.view(-1, Hq, dim), *prompt_exact(*dense, new, total, window=window), f"{extra}, window {window}")


def test_gather_of_many_threads():
    """As many rows as there may be, of 17 heads: 2^31 threads and more for the keys, and as many for the values."""
    heads, dim, page, rows = 17, 16, 256, 1 << 24
    assert (rows // 16 + 2) * heads * 128 > 1 << 31
    c = Cache([page], heads=heads, dim=dim, page=page, seed=3)
    table = torch.full((1, rows // page), int(c.table[0, 0]), dtype=torch.int32, device="cuda")      # every page is the same
    c.max_pages, c.table_dev = rows // page, table
    c.lens_dev.fill_(rows - 3)
    k, v = (torch.full((rows, heads, dim), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
    cg.codegemm_kv_gather(c.struct(), rows, starts([rows]), None, k, v, stream())
    one = [c.k[int(c.table[0, 0])].transpose(0, 1), c.v[int(c.table[0, 0])].permute(1, 3, 0, 2).reshape(page, heads, dim)]
    for got, want in zip((k, v), one):
        got = got.view(rows // page, page, heads, dim)
        assert not bool(got[-1, -3:].any())
        got[-1, -3:] = want[-3:]
        for part in got.split(4096):
            assert bool((part == want).all())
    assert c.intact()

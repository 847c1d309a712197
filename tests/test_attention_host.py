"""Sizes and refusals of the paged cache and the attention calls: host logic, no kernel is launched."""
import ctypes

import pytest

import paper_2512_17970_amd as cg
from paper_2512_17970_amd import binding

INVALID, UNSUPPORTED, TOO_SMALL = -1, -2, -3
AT = 0x10000                                   # an aligned address that nothing is read from


def cache(**kw):
    size = dict(kv_heads=2, head_dim=64, num_pages=8, page_size=32, dtype=binding.KV_INT8, scale_block=16, num_seqs=3, max_pages=4) | {k: v for k, v in kw.items() if k not in POINTERS}
    at = {name: AT for name in POINTERS} | {k: v for k, v in kw.items() if k in POINTERS}
    return cg.KvCache.make(*(at[name] for name in POINTERS), **size)


POINTERS = ("k", "v", "k_scales", "v_scales", "page_table", "kv_lens")


def status(call, *args):
    with pytest.raises(cg.CodegemmError) as e:
        call(*args)
    return e.value.status


def test_structures_are_those_of_the_header(tmp_path):
    """Sizes and offsets of the three structures as a C compiler lays them out."""
    import os
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = {"codegemm_kv_cache": cg.KvCache, "codegemm_append_desc": cg.AppendDesc, "codegemm_attn_desc": cg.AttnDesc}
    lines = [f'printf("{t} %zu\\n", sizeof({t}));' for t in names] + [f'printf("{t}.{f} %zu\\n", offsetof({t}, {f}));' for t, c in names.items() for f, _ in c._fields_]
    src = tmp_path / "s.c"
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"codegemm.h\"\nint main(void) {" + "\n".join(lines) + "return 0; }\n")
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "s")], check=True)
    got = dict(line.rsplit(" ", 1) for line in subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout.splitlines())
    for t, c in names.items():
        assert int(got[t]) == ctypes.sizeof(c)
        for f, _ in c._fields_:
            assert int(got[f"{t}.{f}"]) == getattr(c, f).offset, (t, f)


def test_pool_and_scale_bytes():
    assert cg.codegemm_kv_pool_bytes(cache()) == 8 * 2 * 32 * 64
    assert cg.codegemm_kv_scales_bytes(cache()) == 8 * 2 * 2 * 4
    half = cache(dtype=binding.KV_FP16, scale_block=0)
    assert cg.codegemm_kv_pool_bytes(half) == 8 * 2 * 32 * 64 * 2 and cg.codegemm_kv_scales_bytes(half) == 0
    big = cache(num_pages=1 << 20, kv_heads=8, head_dim=128, page_size=256, scale_block=1)
    assert cg.codegemm_kv_pool_bytes(big) == (1 << 20) * 8 * 256 * 128                     # over 32 bits
    assert cg.codegemm_kv_pool_bytes(cache(k=0, v=0, k_scales=0, v_scales=0, page_table=0, kv_lens=0)) > 0


BAD_CACHES = [(dict(kv_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(num_pages=0), INVALID), (dict(num_seqs=0), INVALID), (dict(max_pages=0), INVALID),
              (dict(head_dim=72), UNSUPPORTED), (dict(head_dim=272), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED),
              (dict(page_size=512), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(scale_block=0), UNSUPPORTED),
              (dict(scale_block=64), UNSUPPORTED), (dict(scale_block=3), UNSUPPORTED), (dict(kv_heads=1025), UNSUPPORTED), (dict(num_seqs=65536), UNSUPPORTED),
              (dict(max_pages=1 << 26), UNSUPPORTED)]


@pytest.mark.parametrize("kw,want", BAD_CACHES)
def test_caches_that_are_refused(kw, want):
    c = cache(**kw)
    assert cg.codegemm_kv_pool_bytes(c) == 0 and cg.codegemm_kv_scales_bytes(c) == 0
    assert status(cg.codegemm_kv_append, c, cg.AppendDesc.make(3, 2), None, AT, AT, AT, None, None, None, AT, None) == want
    assert status(cg.codegemm_kv_gather, c, 4, AT, None, AT, AT) == want
    d = cg.AttnDesc.make(2, 2, 64, num_seqs=3, total_q=3, max_kv=9, scale=1.0)
    assert cg.codegemm_attn_decode_workspace_bytes(c, d) == 0
    assert status(cg.codegemm_attn_decode, c, d, AT, AT, AT, 1 << 30) == want


@pytest.mark.parametrize("name", POINTERS)
def test_pointers_that_are_refused(name):
    for bad in (0, AT + 2):
        c = cache(**{name: bad})
        assert status(cg.codegemm_kv_append, c, cg.AppendDesc.make(3, 2), None, AT, AT, AT, None, None, None, AT, None) == INVALID
        assert status(cg.codegemm_kv_gather, c, 4, AT, None, AT, AT) == INVALID
        assert status(cg.codegemm_attn_decode, c, cg.AttnDesc.make(2, 2, 64, num_seqs=3, total_q=3, max_kv=9, scale=1.0), AT, AT, AT, 1 << 30) == INVALID


def test_appends_that_are_refused():
    def call(desc=None, cu=AT, q=AT, k=AT, v=AT, q_norm=None, k_norm=None, rope=AT, q_out=AT, k_out=None, **kw):
        d = desc or cg.AppendDesc.make(**(dict(tokens=5, q_heads=2, rotary_dim=32, rope_positions=9) | kw))
        return status(cg.codegemm_kv_append, cache(), d, cu, q, k, v, q_norm, k_norm, rope, q_out, k_out)
    for kw in (dict(tokens=0), dict(q_heads=-1), dict(rotary_dim=-16), dict(rotary_dim=80), dict(norm_eps=-1.0), dict(norm_eps=float("nan")), dict(rope_positions=0),
               dict(rope=None), dict(rope=AT + 4), dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(q=AT + 8), dict(k_out=AT + 8), dict(q_norm=AT + 2),
               dict(k_norm=AT + 2), dict(cu=AT + 1), dict(cu=None), dict(q_stride=64), dict(k_stride=132), dict(v_stride=-128), dict(q_out_stride=120), dict(k_out_stride=8),
               dict(k_stride=(1 << 20) + 8)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(tokens=(1 << 24) + 1), dict(q_heads=1025), dict(rotary_dim=24)):
        assert call(**kw) == UNSUPPORTED, kw
    d = cg.AppendDesc.make(5, 2)
    d.flags = 2
    assert call(desc=d) == INVALID


def test_gathers_that_are_refused():
    c = cache()
    for args in ((0, AT, None, AT, AT), (4, None, None, AT, AT), (4, AT + 2, None, AT, AT), (4, AT, AT + 1, AT, AT), (4, AT, None, None, None), (4, AT, None, AT + 8, AT),
                 (4, AT, None, AT, AT + 2)):
        assert status(cg.codegemm_kv_gather, c, *args) == INVALID, args
    assert status(cg.codegemm_kv_gather, c, (1 << 24) + 1, AT, None, AT, AT) == UNSUPPORTED


BAD_ATTENTION = [(dict(q_heads=0), INVALID), (dict(q_heads=3), INVALID), (dict(kv_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(num_seqs=0), INVALID),
                 (dict(total_q=0), INVALID), (dict(total_kv=-1), INVALID), (dict(max_kv=0), INVALID), (dict(window=-1), INVALID), (dict(scale=float("nan")), INVALID),
                 (dict(scale=float("inf")), INVALID), (dict(q_stride=100), INVALID), (dict(k_stride=4), INVALID), (dict(v_stride=129), INVALID), (dict(out_stride=-8), INVALID),
                 (dict(head_dim=40), UNSUPPORTED), (dict(head_dim=512), UNSUPPORTED), (dict(q_heads=2048, kv_heads=2), UNSUPPORTED), (dict(num_seqs=65536), UNSUPPORTED),
                 (dict(total_q=(1 << 24) + 1), UNSUPPORTED), (dict(total_kv=(1 << 24) + 1), UNSUPPORTED)]


def attn(**kw):
    kw = dict(q_heads=4, kv_heads=2, head_dim=64, num_seqs=3, total_q=9, total_kv=9, max_kv=9, scale=0.1) | kw
    return cg.AttnDesc.make(kw.pop("q_heads"), kw.pop("kv_heads"), kw.pop("head_dim"), **kw)


@pytest.mark.parametrize("kw,want", BAD_ATTENTION)
def test_attention_that_is_refused(kw, want):
    assert cg.codegemm_attn_prompt_workspace_bytes(attn(**kw)) == 0
    assert status(cg.codegemm_attn_prompt, attn(**kw), AT, AT, AT, AT, AT, AT, AT, 1 << 40) == want
    single = dict(total_q=3) | kw
    assert cg.codegemm_attn_decode_workspace_bytes(cache(), attn(**single)) == 0
    assert status(cg.codegemm_attn_decode, cache(), attn(**single), AT, AT, AT, 1 << 40) in (want, INVALID)


def test_attention_arguments_that_are_refused():
    need = cg.codegemm_attn_prompt_workspace_bytes(attn())
    assert need > 0
    good = [AT, AT, AT, AT, AT, AT, AT, need]
    for i, bad in [(0, None), (0, AT + 8), (1, None), (2, None), (1, AT + 2), (2, AT + 2), (3, None), (3, AT + 2), (4, AT + 1), (5, None), (5, AT + 4), (6, None), (6, AT + 8)]:
        args = list(good)
        args[i] = bad
        assert status(cg.codegemm_attn_prompt, attn(), *args) == INVALID, (i, bad)
    assert status(cg.codegemm_attn_prompt, attn(total_kv=8), AT, AT, AT, AT, None, AT, AT, need) == INVALID        # one set of lengths, two totals
    assert status(cg.codegemm_attn_prompt, attn(), *good[:7], need - 1) == TOO_SMALL
    d = attn()
    d.flags = 4
    assert status(cg.codegemm_attn_prompt, d, *good) == INVALID
    one = attn(total_q=3)
    need = cg.codegemm_attn_decode_workspace_bytes(cache(), one)
    for args in ((None, AT, AT, need), (AT, None, AT, need), (AT, AT, None, need), (AT + 8, AT, AT, need), (AT, AT + 8, AT, need), (AT, AT, AT + 4, need)):
        assert status(cg.codegemm_attn_decode, cache(), one, *args) == INVALID, args
    assert status(cg.codegemm_attn_decode, cache(), one, AT, AT, AT, need - 1) == TOO_SMALL
    for other in (attn(total_q=3, q_heads=6, kv_heads=3), attn(total_q=3, head_dim=128), attn(total_q=2, num_seqs=2), attn(total_q=4)):
        assert status(cg.codegemm_attn_decode, cache(), other, AT, AT, AT, 1 << 40) == INVALID
    for call in (lambda: cg.load().codegemm_attn_decode(None, None, None, None, None, 0, None), lambda: cg.load().codegemm_attn_prompt(None, *[None] * 7, 0, None),
                 lambda: cg.load().codegemm_kv_append(None, *[None] * 11), lambda: cg.load().codegemm_kv_gather(None, 1, *[None] * 5),
                 lambda: cg.load().codegemm_kv_append(ctypes.byref(cache()), *[None] * 11)):
        assert call() == INVALID


def test_decode_workspace():
    """Fixed areas, and [16][D + 2] sums for two pieces of an item for every workgroup that runs at once: 256, 512 where there are more items, fewer
    where there is less to do."""
    fixed, each = 65536 + (2 << 20), 2 * 16 * 66 * 4
    need = lambda seqs, keys, **kw: cg.codegemm_attn_decode_workspace_bytes(cache(num_seqs=seqs, max_pages=4000), attn(num_seqs=seqs, total_q=seqs, max_kv=keys, **kw))  # noqa: E731
    assert need(600, 3000) == fixed + 512 * each and need(129, 10) == fixed + 258 * each
    assert need(1, 100000) == need(128, 3000) == fixed + 256 * each
    assert fixed + 2 * each <= need(1, 100) < need(1, 3000) < fixed + 256 * each
    assert need(1, 100000, window=100) == need(1, 100)
    assert need(1, 100000, window=1 << 30) == fixed + 256 * each


def test_lengths_that_the_host_does_not_know():
    """Any max_kv: what is split is bounded by the keys that there can be."""
    most = (1 << 31) - 1
    for total in (0, 1, 100, 5000, 1 << 24):
        need = [cg.codegemm_attn_prompt_workspace_bytes(attn(q_heads=8, kv_heads=8, num_seqs=1, total_q=16, total_kv=total, max_kv=n, window=w)) for n in (1 << 24, most) for w in (0, most)]
        assert len(set(need)) == 1 and 0 < need[0] < 64 << 20
    single = dict(num_seqs=3, total_q=3)
    need = [cg.codegemm_attn_decode_workspace_bytes(cache(max_pages=m), attn(max_kv=n, window=w, **single)) for m in (1000, 1 << 25) for n in (32000, most) for w in (0, most)]
    assert all(x > 0 for x in need) and need[0] == need[1] == need[2] == need[3]


def test_launches_that_are_too_large():
    """2^32 threads and more are refused, not sent."""
    c = cache(kv_heads=1024, head_dim=16, num_pages=1 << 30)
    d = attn(q_heads=1024, kv_heads=1024, head_dim=16, total_q=1 << 24, total_kv=1 << 24)
    assert cg.codegemm_attn_prompt_workspace_bytes(d) == 0 and status(cg.codegemm_attn_prompt, d, *[AT] * 7, 1 << 40) == UNSUPPORTED
    assert status(cg.codegemm_kv_append, c, cg.AppendDesc.make(1 << 24, 0), AT, None, AT, AT, None, None, None, None, None) == UNSUPPORTED
    assert status(cg.codegemm_kv_gather, c, 1 << 24, AT, None, AT, AT) == UNSUPPORTED

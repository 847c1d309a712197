"""Sizes and refusals of the calls that sum attention weights and evict: host logic, no kernel is launched."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2512_17970_amd as cg
from test_attention_host import AT, BAD_ATTENTION, BAD_CACHES, INVALID, TOO_SMALL, UNSUPPORTED, attn, cache, status

FIXED = 65536 + (2 << 20)


def single(**kw):
    return attn(**(dict(total_q=3) | kw))


def test_the_structure_is_that_of_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = ["sizeof(codegemm_evict_desc)"] + [f"offsetof(codegemm_evict_desc, {f})" for f, _ in cg.EvictDesc._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "codegemm.h"\nint main(void) {' + "".join(f'printf("%zu\\n", {x});' for x in lines) + "return 0; }\n")
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "s")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(cg.EvictDesc)] + [getattr(cg.EvictDesc, f).offset for f, _ in cg.EvictDesc._fields_]


@pytest.mark.parametrize("kw,want", BAD_CACHES)
def test_caches_that_are_refused(kw, want):
    c = cache(**kw)
    e = cg.EvictDesc.make(5, max_kv=9)
    assert cg.codegemm_attn_scores_workspace_bytes(c, single()) == cg.codegemm_attn_decode_scores_workspace_bytes(c, single()) == cg.codegemm_kv_evict_workspace_bytes(c, e) == 0
    assert status(cg.codegemm_attn_scores, c, single(), AT, None, None, None, AT, AT, 1 << 40) == want
    assert status(cg.codegemm_attn_decode_scores, c, single(), AT, AT, None, None, AT, AT, 1 << 40) == want
    assert status(cg.codegemm_kv_evict, c, cache(), e, AT, None, None, AT, None, AT, 1 << 40) == want
    assert status(cg.codegemm_kv_evict, cache(), c, e, AT, None, None, AT, None, AT, 1 << 40) == want


@pytest.mark.parametrize("kw,want", BAD_ATTENTION)
def test_scores_that_are_refused(kw, want):
    d = single(**kw)
    assert cg.codegemm_attn_scores_workspace_bytes(cache(), d) == cg.codegemm_attn_decode_scores_workspace_bytes(cache(), d) == 0 or "total_kv" in kw or "k_stride" in kw
    assert status(cg.codegemm_attn_scores, cache(), d, AT, AT, None, None, AT, AT, 1 << 40) in (want, INVALID)
    assert status(cg.codegemm_attn_decode_scores, cache(), d, AT, AT, None, None, AT, AT, 1 << 40) in (want, INVALID)


def test_arguments_of_scores_that_are_refused():
    need = cg.codegemm_attn_scores_workspace_bytes(cache(), attn())
    good = [AT, AT, AT, AT, AT, AT, need]
    for i, bad in [(0, None), (0, AT + 8), (1, AT + 2), (1, None), (2, AT + 1), (3, AT + 4), (4, None), (4, AT + 4), (5, None), (5, AT + 8)]:
        args = list(good)
        args[i] = bad
        assert status(cg.codegemm_attn_scores, cache(), attn(), *args) == INVALID, (i, bad)          # (no cu_q: nine queries, three sequences)
    assert status(cg.codegemm_attn_scores, cache(), attn(), *good[:6], need - 1) == TOO_SMALL
    need = cg.codegemm_attn_decode_scores_workspace_bytes(cache(), single())
    good = [AT, AT, AT, AT, AT, AT, need]
    for i, bad in [(0, None), (0, AT + 8), (1, None), (1, AT + 2), (2, AT + 1), (3, AT + 4), (4, None), (4, AT + 4), (5, None), (5, AT + 8)]:
        args = list(good)
        args[i] = bad
        assert status(cg.codegemm_attn_decode_scores, cache(), single(), *args) == INVALID, (i, bad)
    assert status(cg.codegemm_attn_decode_scores, cache(), single(), *good[:6], need - 1) == TOO_SMALL
    assert cg.codegemm_attn_decode_scores_workspace_bytes(cache(), attn()) == 0 and status(cg.codegemm_attn_decode_scores, cache(), attn(), *good[:6], 1 << 40) == INVALID
    for other in (single(q_heads=6, kv_heads=3), single(head_dim=128), single(total_q=2, num_seqs=2)):
        assert status(cg.codegemm_attn_scores, cache(), other, AT, AT, None, None, AT, AT, 1 << 40) == INVALID
    lib = cg.load()
    assert lib.codegemm_attn_scores(None, None, *[None] * 6, 0, None) == lib.codegemm_attn_decode_scores(None, None, *[None] * 6, 0, None) == INVALID
    assert lib.codegemm_attn_scores(ctypes.byref(cache()), None, *[None] * 6, 0, None) == INVALID


def test_workspace_of_scores():
    """Rows' sums of 8 bytes, in parts for what shares the keys; beyond what is worth it, more rows have no more parts."""
    rows = lambda n: (n * 4 * 8 + 255) // 256 * 256  # noqa: E731
    assert cg.codegemm_attn_scores_workspace_bytes(cache(), attn(max_kv=100)) == FIXED + rows(9) + 9 * 4 * 8
    long = cache(max_pages=10000)
    one = cg.codegemm_attn_scores_workspace_bytes(long, attn(total_q=9, max_kv=100000))
    parts = -(-512 // (long.num_seqs * long.kv_heads))                     # 512 workgroups between sequences and key heads, fewer than there are blocks of 256 keys
    assert parts < -(-100000 // 256) and one == FIXED + rows(9) + parts * 9 * 4 * 8
    assert cg.codegemm_attn_scores_workspace_bytes(long, attn(total_q=1 << 24, max_kv=100000)) == FIXED + 2 * rows(1 << 24)
    assert cg.codegemm_attn_scores_workspace_bytes(cache(), attn(max_kv=(1 << 31) - 1)) == cg.codegemm_attn_scores_workspace_bytes(cache(), attn(max_kv=128))
    assert cg.codegemm_attn_decode_scores_workspace_bytes(cache(), single()) >= cg.codegemm_attn_decode_workspace_bytes(cache(), single()) + 3 * 4 * 8


BAD_EVICTIONS = [dict(budget=0), dict(budget=-4), dict(keep_first=-1), dict(keep_last=-1), dict(keep_first=6), dict(keep_first=3, keep_last=3), dict(keep_first=(1 << 31) - 1, keep_last=5),
                 dict(max_kv=0)]


@pytest.mark.parametrize("kw", BAD_EVICTIONS)
def test_evictions_that_are_refused(kw):
    e = cg.EvictDesc.make(**(dict(budget=5, max_kv=9) | kw))
    assert cg.codegemm_kv_evict_workspace_bytes(cache(), e) == 0
    assert status(cg.codegemm_kv_evict, cache(), cache(), e, AT, None, None, AT, None, AT, 1 << 40) == INVALID


def test_arguments_of_evictions_that_are_refused():
    e = cg.EvictDesc.make(5, max_kv=9)
    need = cg.codegemm_kv_evict_workspace_bytes(cache(), e)
    assert need == FIXED + (3 * 2 * 5 * 4 + 255) // 256 * 256 + 3 * 2 * 8
    good = [AT, AT, AT, AT, AT, AT, need]
    for i, bad in [(0, None), (0, AT + 4), (1, AT + 2), (2, AT + 4), (3, None), (3, AT + 1), (4, AT + 2), (5, None), (5, AT + 8)]:
        args = list(good)
        args[i] = bad
        assert status(cg.codegemm_kv_evict, cache(), cache(), e, *args) == INVALID, (i, bad)
    assert status(cg.codegemm_kv_evict, cache(), cache(), e, *good[:6], need - 1) == TOO_SMALL
    for other in (dict(kv_heads=1), dict(head_dim=128), dict(page_size=64), dict(dtype=cg.KV_FP8), dict(scale_block=8), dict(num_seqs=2)):
        assert status(cg.codegemm_kv_evict, cache(), cache(**other), e, *good) == INVALID, other
    for name in ("k", "v", "k_scales", "v_scales", "page_table", "kv_lens"):
        for pair in ((cache(**{name: 0}), cache()), (cache(), cache(**{name: AT + 2}))):
            assert status(cg.codegemm_kv_evict, *pair, e, *good) == INVALID
    lib = cg.load()
    assert lib.codegemm_kv_evict(None, None, None, *[None] * 6, 0, None) == INVALID
    assert lib.codegemm_kv_evict(ctypes.byref(cache()), None, ctypes.byref(e), *[None] * 6, 0, None) == INVALID
    assert lib.codegemm_kv_evict(ctypes.byref(cache()), ctypes.byref(cache()), None, *[None] * 6, 0, None) == INVALID


def test_launches_that_are_too_large():
    c = cache(kv_heads=1024, num_seqs=65535, num_pages=1 << 30)
    assert cg.codegemm_kv_evict_workspace_bytes(c, cg.EvictDesc.make(5, max_kv=9)) == 0
    assert status(cg.codegemm_kv_evict, c, c, cg.EvictDesc.make(5, max_kv=9), AT, None, None, AT, None, AT, 1 << 60) == UNSUPPORTED
    d = attn(q_heads=1024, kv_heads=1024, num_seqs=65535, total_q=65535)
    assert cg.codegemm_attn_scores_workspace_bytes(c, d) == 0 and status(cg.codegemm_attn_scores, c, d, AT, None, None, None, AT, AT, 1 << 60) == UNSUPPORTED
    assert cg.codegemm_attn_scores_workspace_bytes(cache(), attn(q_heads=64, kv_heads=2, total_q=1 << 24)) > 0
    assert cg.codegemm_attn_scores_workspace_bytes(cache(), attn(q_heads=66, kv_heads=2, total_q=1 << 24)) == 0
    d = attn(q_heads=1024, kv_heads=2, total_q=1 << 24)
    assert cg.codegemm_attn_scores_workspace_bytes(cache(), d) == 0 and status(cg.codegemm_attn_scores, cache(), d, AT, AT, None, None, AT, AT, 1 << 60) == UNSUPPORTED

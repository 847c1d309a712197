"""Sizes and refusals of the cache in 4 bits: host logic, no kernel is launched."""
import pytest

import paper_2512_17970_amd as cg
from test_attention_host import AT, INVALID, UNSUPPORTED, cache, status


def four(**kw):
    return cache(**(dict(dtype=cg.KV_INT4, scale_block=32) | kw))


def test_pool_and_scale_bytes():
    assert cg.codegemm_kv_pool_bytes(four()) == 8 * 2 * 32 * 64 // 2 and cg.codegemm_kv_scales_bytes(four()) == 8 * 2 * 32 * 2 * 4
    assert cg.codegemm_kv_scales_bytes(four(scale_block=256)) == 8 * 2 * 32 * 4                     # one run for a head
    assert cg.codegemm_kv_scales_bytes(four(head_dim=96, scale_block=64)) == 8 * 2 * 32 * 2 * 4     # the second of them shorter
    big = four(num_pages=1 << 20, kv_heads=8, head_dim=128, page_size=256)
    assert cg.codegemm_kv_pool_bytes(big) == (1 << 20) * 8 * 256 * 64 and cg.codegemm_kv_scales_bytes(big) == (1 << 20) * 8 * 256 * 16


@pytest.mark.parametrize("kw", [dict(head_dim=16), dict(head_dim=80), dict(scale_block=0), dict(scale_block=1), dict(scale_block=16), dict(scale_block=48), dict(scale_block=512),
                                dict(dtype=3), dict(dtype=5)])
def test_caches_that_are_refused(kw):
    c = four(**kw)
    assert cg.codegemm_kv_pool_bytes(c) == 0 and cg.codegemm_kv_scales_bytes(c) == 0
    assert status(cg.codegemm_kv_append, c, cg.AppendDesc.make(3, 2), None, AT, AT, AT, None, None, None, AT, None) == UNSUPPORTED
    assert status(cg.codegemm_kv_gather, c, 4, AT, None, AT, AT) == UNSUPPORTED
    d = cg.AttnDesc.make(2, 2, c.head_dim, num_seqs=3, total_q=3, max_kv=9, scale=1.0)
    assert cg.codegemm_attn_decode_workspace_bytes(c, d) == 0 and status(cg.codegemm_attn_decode, c, d, AT, AT, AT, 1 << 30) == UNSUPPORTED


def test_pointers_that_are_refused():
    for name in ("k", "v", "k_scales", "v_scales", "page_table", "kv_lens"):
        for bad in (0, AT + 2):
            c = four(**{name: bad})
            assert status(cg.codegemm_kv_append, c, cg.AppendDesc.make(3, 2), None, AT, AT, AT, None, None, None, AT, None) == INVALID
            assert status(cg.codegemm_kv_gather, c, 4, AT, None, AT, AT) == INVALID


def test_shifted_appends_that_are_refused():
    args = [None, AT, AT, AT, None, None, None, AT, None]
    assert status(cg.codegemm_kv_append_shifted, four(), cg.AppendDesc.make(3, 2), None, AT + 2, *args[1:]) == INVALID
    assert status(cg.codegemm_kv_append_shifted, four(), cg.AppendDesc.make(0, 2), None, AT, *args[1:]) == INVALID
    assert status(cg.codegemm_kv_append_shifted, four(head_dim=80), cg.AppendDesc.make(3, 2), None, AT, *args[1:]) == UNSUPPORTED
    assert cg.load().codegemm_kv_append_shifted(None, *[None] * 12) == INVALID

"""What the calls that sum attention weights refuse, each with its status: host logic, no kernel is launched."""
import pytest

import paper_2512_17970_amd as cg
from test_attention_host import AT, BAD_ATTENTION, attn, cache, status


@pytest.mark.parametrize("kw,want", BAD_ATTENTION)
def test_each_has_its_status_and_no_workspace(kw, want):
    """total_kv and strides that the calls have no use for among them."""
    for total in (3, 9):
        d = attn(**(dict(total_q=total) | kw))
        assert cg.codegemm_attn_scores_workspace_bytes(cache(), d) == 0
        assert status(cg.codegemm_attn_scores, cache(), d, AT, AT, None, None, AT, AT, 1 << 40) == want
    d = attn(**(dict(total_q=3) | kw))
    assert cg.codegemm_attn_decode_scores_workspace_bytes(cache(), d) == 0
    assert status(cg.codegemm_attn_decode_scores, cache(), d, AT, AT, None, None, AT, AT, 1 << 40) == want


def test_what_is_not_used_makes_no_difference():
    for size in (cg.codegemm_attn_scores_workspace_bytes, cg.codegemm_attn_decode_scores_workspace_bytes):
        want = size(cache(), attn(total_q=3))
        assert want > 0 and all(size(cache(), attn(total_q=3, **kw)) == want for kw in (dict(total_kv=0), dict(total_kv=1 << 24), dict(k_stride=136), dict(v_stride=1 << 20), dict(out_stride=264)))

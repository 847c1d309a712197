"""Attention with scores where there are more sequences and key heads than compute units: two workgroups share a unit then."""
import pytest
import torch

pytestmark = pytest.mark.gpu

cg = pytest.importorskip("paper_2512_17970_amd")
from attention_util import check, decode_exact  # noqa: E402
from test_gpu_attention_scores import FP16, FP8, INT4, INT8, make, queries, run  # noqa: E402

LENS = [97, 1, 0, 40, 16, 33, 64, 5] + [3, 18] * 22


@pytest.mark.parametrize("dtype,block", [(FP16, 1), (INT8, 1), (INT8, 16), (FP8, 4), (INT4, 32)])
@pytest.mark.parametrize("heads,group,dim,window", [(5, 1, 64, 0), (5, 2, 128, 20), (5, 1, 96, 0), (3, 17, 64, 20), (5, 1, 256, 0)])
def test_more_than_compute_units(dtype, block, heads, group, dim, window):
    c = make(LENS, dtype, heads=heads, dim=dim, block=block, page=32, seed=dim)
    q = queries(len(LENS), heads * group, dim)
    _, out = run(c, q, [1] * len(LENS), single=True, window=window)
    if dtype == INT4:
        from test_gpu_four_bits import decode_exact as exact4
        check(out, *exact4(c, q, window=window), "out")
    else:
        check(out, *decode_exact(c, q, window=window), "out")

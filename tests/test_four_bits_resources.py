"""Registers and spills of the kernels of the cache in 4 bits, of the scores and of eviction, as the number of wavefronts that they were laid out for allows them."""
import pytest

pytest.importorskip("msgpack")
from test_attention_resources import of  # noqa: E402
from test_kernel_resources import _kernels  # noqa: E402


@pytest.fixture(scope="module")
def kernels():
    return _kernels()


# Up to 12 wavefronts of a compute unit for heads of 64, eight for 128, four for 256.
@pytest.mark.parametrize("dim,registers", [(64, 168), (128, 256), (256, 512)])
def test_single_tokens(kernels, dim, registers):
    found = of(kernels, "attn_decode_kernel", 4, dim)
    assert len(found) == 4 and all(r <= registers and s == 0 for r, s in found), found


@pytest.mark.parametrize("name,registers", [("kv_append_kernel", 128), ("kv_gather_kernel", 64)])
def test_cache(kernels, name, registers):
    assert all(r <= registers and s == 0 for r, s in of(kernels, name, 4))


# Scores of many rows: two wavefronts on a SIMD.  Codes of 8 bits and heads of less than 128 spill values that stay the same through the loops.
@pytest.mark.parametrize("name", ["score_stats_kernel", "score_sum_kernel"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind", [0, 1, 2, 4])
def test_scores(kernels, name, dim, kind):
    spills = 48 if dim == 128 and kind != 4 else 2
    assert all(r <= 256 and s <= spills for r, s in of(kernels, name, kind, dim))


# .. of few: three, for wide codes two.
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind", [0, 1, 2, 4])
def test_scores_of_few_rows(kernels, dim, kind):
    assert all(r <= (256 if kind == 0 else 168) and s <= (10 if kind in (1, 2) else 0) for r, s in of(kernels, "score_few_kernel", kind, dim))


# A workgroup of 1024 threads; five of 256 on a compute unit.
def test_eviction(kernels):
    for name in [f"kv_select_part_kernelILi{i}E" for i in range(4)] + ["kv_select_kernelE"]:
        assert all(v[0] <= 128 and v[1] == 0 for k, v in kernels.items() if name in k) and any(name in k for k in kernels), name
    for kind in (0, 1, 2, 4):
        assert all(r <= 96 and s == 0 for r, s in of(kernels, "kv_move_kernel", kind))

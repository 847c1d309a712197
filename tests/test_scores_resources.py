"""Spilled registers of the kernels of attention's scores, instance by instance: where they are none now, and how many at most elsewhere."""
import pytest

pytest.importorskip("msgpack")
from test_attention_resources import of  # noqa: E402
from test_kernel_resources import _kernels  # noqa: E402

# (kernel, type of the cache, dimensions that heads are worked on as) -> spills of heads of exactly these dimensions, and of smaller ones
SPILLS = {("score_stats_kernel", 1, 128): (14, 29), ("score_stats_kernel", 2, 128): (12, 27), ("score_sum_kernel", 0, 128): (0, 12),
          ("score_few_kernel", 1, 128): (0, 8), ("score_few_kernel", 2, 128): (0, 7), ("score_few_kernel", 1, 256): (0, 10)}


@pytest.fixture(scope="module")
def kernels():
    return _kernels()


@pytest.mark.parametrize("name", ["score_stats_kernel", "score_sum_kernel", "score_few_kernel"])
@pytest.mark.parametrize("kind", [0, 1, 2, 4])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_spills(kernels, name, kind, dim):
    for exact, most in zip((1, 0), SPILLS.get((name, kind, dim), (0, 0))):
        (_, spills), = of(kernels, name, kind, f"{dim}ELb{exact}")
        assert spills <= most, (exact, spills)

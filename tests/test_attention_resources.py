"""Registers and spills of the kernels of the cache and of attention, as the number of wavefronts that they were laid out for allows them: 512 registers of a SIMD."""
import pytest

pytest.importorskip("msgpack")
from test_kernel_resources import _kernels  # noqa: E402


@pytest.fixture(scope="module")
def kernels():
    return _kernels()


def of(kernels, name, *first):
    """(registers, spills) of every instance of a kernel whose first template arguments these are."""
    start = f"{len(name)}{name}ILi" + "ELi".join(map(str, first))
    found = [v[:2] for k, v in kernels.items() if start + "E" in k]
    assert found, start
    return found


# Heads of up to 64: three wavefronts of 168 registers; of 128: two; of 256: one, of which 7 do not fit.
@pytest.mark.parametrize("dim,registers,spills", [(64, 168, 0), (128, 256, 0), (256, 512, 7)])
def test_prompts(kernels, dim, registers, spills):
    found = of(kernels, "attn_prompt_kernel", dim)
    assert len(found) == 2 and all(r <= registers and s <= spills for r, s in found), found


# Eight wavefronts of a compute unit, four for those whose two steps in LDS leave no room for more.
@pytest.mark.parametrize("kind,dim,registers", [(0, 64, 256), (0, 128, 512), (0, 256, 512), (1, 64, 256), (1, 128, 256), (1, 256, 512), (2, 64, 256), (2, 128, 256), (2, 256, 512)])
def test_single_tokens(kernels, kind, dim, registers):
    assert all(r <= registers and s == 0 for r, s in of(kernels, "attn_decode_kernel", kind, dim))


# Appending: 16 wavefronts of a compute unit; a gather has as many as there are.
@pytest.mark.parametrize("name,registers", [("kv_append_kernel", 128), ("kv_gather_kernel", 64)])
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_cache(kernels, name, registers, kind):
    assert all(r <= registers and s == 0 for r, s in of(kernels, name, kind))

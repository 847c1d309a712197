import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


def _skip_tests_of_the_extension(items):
    # The binding does without its extension module where that cannot be built; so do the tests.  Where it could be, a missing one is an error.
    from paper_2512_17970_amd import binding, build
    if binding._calls is not None or build.can_build_calls():
        return
    skip = pytest.mark.skip(reason="no extension module, and no g++ or Python.h to build it with")
    for item in items:
        if "calls" in getattr(item, "fixturenames", ()) or item.name == "test_the_module_exports_the_extension":
            item.add_marker(skip)


def pytest_collection_modifyitems(config, items):
    _skip_tests_of_the_extension(items)
    # GPU tests are skipped, loudly, when no device is present, so a plain
    # `pytest tests/` on a CPU machine does not fail.
    try:
        import torch
        have_gpu = torch.cuda.is_available()
    except Exception:
        have_gpu = False
    if have_gpu:
        return
    skip = pytest.mark.skip(reason="no GPU in this environment")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)

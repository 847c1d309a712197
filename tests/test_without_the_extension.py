"""The tests of the extension module's calls where there is neither the module nor a compiler for it: skipped, not failed."""
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.parametrize("compiler", [False, True])
def test_tests_of_the_extension(tmp_path, compiler):
    (tmp_path / "no_extension.py").write_text('import sys\nsys.modules["paper_2512_17970_amd._calls"] = None\n')
    if compiler:
        (tmp_path / "g++").write_text("")
        (tmp_path / "g++").chmod(0o755)
    env = {**os.environ, "PYTHONPATH": str(tmp_path), "PATH": str(tmp_path)}
    files = [os.path.join(HERE, f"test_python_calls{which}.py") for which in ("", "_attention")]
    got = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no_extension", "-p", "no:cacheprovider", *files, "-k", "raises or exports"], cwd=os.path.dirname(HERE),
                         env=env, capture_output=True, text=True, timeout=100)
    summary = got.stdout.splitlines()[-1]
    if compiler:                                     # it could have been built, so its absence is an error
        assert got.returncode == 1 and "error" in summary, summary
    else:
        assert got.returncode == 0 and "skipped" in summary and "error" not in summary and "failed" not in summary, got.stdout[-2000:]

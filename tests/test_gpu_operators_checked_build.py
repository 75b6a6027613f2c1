"""The tests of the operators around the cache in the checked build (see test_gpu_checked_build.py), in a child process."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(os.environ.get("HACK_B200_CHECKED", "0") == "1", reason="this is the child process")
def test_operators_in_the_checked_build():
    import __graft_entry__ as ge
    ge.build()
    files = ["tests/test_gpu_kv4.py", "tests/test_gpu_rope.py", "tests/test_gpu_operator_edges.py"]
    res = subprocess.run([sys.executable, "-m", "pytest", "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider"] + files, cwd=ROOT,
                         env=dict(os.environ, HACK_B200_CHECKED="1"), capture_output=True, text=True, timeout=900)
    tail = "\n".join((res.stdout + res.stderr).splitlines()[-25:])
    assert res.returncode == 0, tail
    assert " passed" in res.stdout and "no tests ran" not in res.stdout, tail

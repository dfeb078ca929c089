"""The tests of the messages on the debug build (bounds-checked kernels), in a child process that loads it: same results,
and no access out of the callers' buffers, the arenas and the scratch.  (No test provokes one on the GPU.)"""
import os
import subprocess
import sys

import pytest

from gpu_common import require_gpu

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))


def test_messages_on_the_debug_build():
    require_gpu()
    if os.environ.get("HADFL_LIBRARY"):
        pytest.skip("already running inside a child process with a library of its own")
    from paper_2111_08274_b200 import build
    env = dict(os.environ, HADFL_LIBRARY=build.build(debug=True))
    targets = [os.path.join(HERE, f) for f in ("test_gpu_packed.py", "test_gpu_packed_run.py")]
    got = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", *targets],
                         cwd=os.path.dirname(HERE), env=env, capture_output=True, text=True)
    assert got.returncode == 0, got.stdout[-4000:] + got.stderr[-2000:]

"""The longer tests of the messages on the debug build (bounds-checked kernels), in a child process that loads it."""
import os
import subprocess
import sys

import pytest

from gpu_common import require_gpu

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
FILES = ["test_gpu_packed_order.py", "test_gpu_packed_rows.py", "test_gpu_packed_capture.py", "test_gpu_packed_products.py"]


def test_longer_messages_on_the_debug_build():
    require_gpu()
    if os.environ.get("HADFL_LIBRARY"):
        pytest.skip("already running inside a child process with a library of its own")
    from paper_2111_08274_b200 import build
    env = dict(os.environ, HADFL_LIBRARY=build.build(debug=True))
    got = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider",
                          *(os.path.join(HERE, f) for f in FILES)], cwd=os.path.dirname(HERE), env=env, capture_output=True, text=True)
    assert got.returncode == 0, got.stdout[-4000:] + got.stderr[-2000:]

"""What has to hold of the messages' kernels by their source, where a fault would be a hang or a race on the GPU that no
run is sure to show (csrc/packed.cuh is read as text)."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def source():
    text = open(os.path.join(ROOT, "paper_2111_08274_b200", "csrc", "packed.cuh")).read()
    return re.sub(r"//[^\n]*", "", text)


def test_lanes_are_together_before_aligned_instructions_on_tensor_memory(source):
    """tcgen05.alloc, .ld and .dealloc are undefined (they may hang) when a warp's lanes are apart, as they may be behind a
    wait, a loop or a branch of each lane: a __syncwarp() comes directly before."""
    found = [m for m in re.finditer(r'asm volatile\(\s*"tcgen05\.(alloc|ld|dealloc)\b', source)]
    assert sorted(m[1] for m in found) == ["alloc", "dealloc", "ld"]
    assert len(found) == len(re.findall(r"tcgen05\.(?:alloc|ld|dealloc)\b", source))
    for m in found:
        assert source[:m.start()].rstrip().endswith("__syncwarp();"), m[1]


def test_inputs_are_read_coherently(source):
    """The kernels may be on the GPU while the one before them in the stream still writes what they are going to read.  A
    const __restrict__ pointer promises that nobody does, and allows loads through the read-only path or ahead of the wait."""
    kernels = re.findall(r"__global__ void\s+__launch_bounds__\((?:[^()]|\([^()]*\))*\)\s*(k_\w+)\(([^)]*)\)", source)
    assert len(kernels) == source.count("__global__") == 5
    for name, arguments in kernels:
        assert "__restrict__" not in arguments, name
    assert not re.search(r"__ldg\b|\.nc\b", source)

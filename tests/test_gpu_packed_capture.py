"""Messages in CUDA graphs: captured as the first calls of a process, and behind copies, fills, events and other kernels
(the launches ask for an early start, which a graph knows between kernels only)."""
import os
import subprocess
import sys

import pytest
import torch

from gpu_common import require_gpu
from paper_2111_08274_b200 import binding
from test_gpu_packed import Side

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


FIRST = """
import torch
from paper_2111_08274_b200 import binding
n, p = 4, 20_003
stream = torch.cuda.Stream()
stride = -(-p // 32) * 32
w = torch.randn((n, stride), device="cuda")
start = w.clone()
m, base = torch.zeros_like(w), torch.zeros(p, device="cuda")
messages = torch.zeros((n, binding.hadfl_packed_bytes(p)), dtype=torch.uint8, device="cuda")
outs = torch.zeros((2, n, n), device="cuda")
h = binding.Hadfl(n, p, w_ptr=w.data_ptr(), m_ptr=m.data_ptr(), row_stride_elems=stride, stream=stream.cuda_stream)
torch.cuda.synchronize()
w.copy_(start)
torch.cuda.synchronize()

def calls(out):
    h.pack(range(n), messages.data_ptr(), base_ptr=base.data_ptr())
    h.packed_dots(range(n), messages.data_ptr(), out.data_ptr())
    h.packed_dots(range(n), messages.data_ptr(), out.data_ptr(), b_ids=range(n - 1, -1, -1), b_messages_ptr=messages.data_ptr())
    h.unpack([3], messages.data_ptr())
    h.aggregate_packed([0, 1], messages.data_ptr(), base_ptr=base.data_ptr())
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=stream):
    calls(outs[0])
with torch.cuda.stream(stream):
    graph.replay()
torch.cuda.synchronize()
got = w.clone()
w.copy_(start)
torch.cuda.synchronize()
calls(outs[1])
torch.cuda.synchronize()
assert torch.equal(got, w) and torch.equal(outs[0], outs[1]) and bool((outs[0].flip(1).diagonal() > 0).all())
print("captured first")
"""


def test_captured_before_any_call():
    if binding.hadfl_debug_build():
        pytest.skip("the debug build wants a call with each buffer before it is captured")
    got = subprocess.run([sys.executable, "-c", FIRST], cwd=ROOT, capture_output=True, text=True)
    assert got.returncode == 0 and "captured first" in got.stdout, got.stdout[-2000:] + got.stderr[-4000:]


def events(stream, other, work):
    """`work` on another stream that begins when `stream` is here, and that it waits for."""
    e = torch.cuda.Event()
    e.record(stream)
    other.wait_event(e)
    with torch.cuda.stream(other):
        work()
    e = torch.cuda.Event()
    e.record(other)
    stream.wait_event(e)


@pytest.mark.parametrize("n,p", [(3, 1003), (8, 300_007)])
@pytest.mark.parametrize("before", ["copy", "fill", "event", "two streams", "kernel"])
def test_captured_behind_other_work(n, p, before):
    """Before every call the parameters come anew, by what `before` says; replays give what the calls give."""
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    g = torch.Generator(device="cuda").manual_seed(n)
    s = Side(n, p, stream=stream)
    source = 1e-2 * torch.randn(s.w.shape, generator=g, device="cuda")
    base, out = torch.zeros(p, device="cuda"), torch.zeros((n, n), device="cuda")
    ids = list(range(n))
    torch.cuda.synchronize()

    def anew(to, value):
        if before == "copy":
            to.copy_(value, non_blocking=True)
        elif before == "fill":
            to.zero_()
            to[:, ::2].add_(value[:, ::2])
            to.view(torch.uint8)[:, -1].fill_(0)
        elif before == "event":
            events(stream, other, lambda: to.copy_(value, non_blocking=True))
        elif before == "two streams":
            events(stream, other, lambda: to[0].copy_(value[0]))
            to[1:].copy_(value[1:])
        else:
            torch.mul(value, 1.5, out=to)

    def calls():
        anew(s.w, source)
        s.h.pack(ids, s.messages.data_ptr(), base_ptr=base.data_ptr(), residual_ptr=s.residual.data_ptr(), round_=1)
        anew(s.m, source)
        s.h.packed_dots(ids, s.messages.data_ptr(), out.data_ptr())
        anew(s.residual, source)
        s.h.aggregate_packed(ids[:2], s.messages.data_ptr(), base_ptr=base.data_ptr(), dst_ids=ids[1:], move_base=True)
        anew(s.m, source)
        s.h.unpack(ids[:1], s.messages.data_ptr(), base_ptr=base.data_ptr())

    def state():
        torch.cuda.synchronize()
        return [t.clone() for t in (s.w, s.residual, s.messages, base, out)]

    def reset():
        torch.cuda.synchronize()
        base.zero_()
        s.residual.zero_()
        out.zero_()
        torch.cuda.synchronize()
    reset()
    want = []
    for _ in range(3):
        with torch.cuda.stream(stream):
            calls()
        want.append(state())
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        calls()
    reset()
    for r in range(3):
        with torch.cuda.stream(stream):
            graph.replay()
        for x, y in zip(state(), want[r]):
            assert torch.equal(x, y), r
    assert bool((want[2][4].diagonal() > 0).all())
    s.h.debug_check()

"""A process whose first calls of the recurrent core are captured: kernel attributes and tensor maps are made while a stream is recorded."""
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

PROGRAM = """
import torch, paper_2012_09849_b200 as hts
g = torch.Generator(device="cuda").manual_seed(1)
r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
T, N, D, S = 40, 3, 64, 16
x, dt, b, c, w, dy = r(T, N, D), r(T, N, D), r(T, N, S), r(T, N, S), r(512, D), r(T, N, D)
a, taps = -torch.rand(D, S, device="cuda"), torch.rand(D, 4, device="cuda")
work = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (hts.hts_selective_scan_workspace(T, N, D, S) + 16, hts.hts_selective_scan_workspace(T, N, D, S, True),
        hts.hts_causal_conv_workspace(T, N, D, 4), hts.hts_linear_workspace(T * N, D, 512), hts.hts_linear_workspace(T * N, D, 512, True), hts.hts_linear_workspace(4000, D, 512))]
big = r(4000, D)
def out():
    return [torch.zeros(T, N, D, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(x), torch.zeros_like(x), torch.zeros(T * N, 512, dtype=torch.bfloat16, device="cuda"),
            torch.zeros(512, D, device="cuda"), torch.zeros(4000, 512, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(x)]
def calls(o):
    hts.hts_causal_conv(x, taps, None, None, None, None, "silu", o[0], None)
    hts.hts_selective_scan(x, dt, a, b, c, None, None, None, None, None, None, True, o[1], None, work[0])
    hts.hts_selective_scan_gradient(x, dt, a, b, c, None, None, None, None, None, None, True, dy, None, {"x": o[2]}, work[1])
    hts.hts_linear(x.view(T * N, D), w, None, None, "relu", o[3], None, work[3])
    hts.hts_linear_gradient(x.view(T * N, D), w, None, o[3], "none", None, o[4], None, work[4])
    hts.hts_linear(big, w, None, None, "none", o[5], None, work[5])
    hts.hts_causal_conv_gradient(x, taps, None, None, None, None, "silu", dy, None, o[6], None, None, None, work[2])
first, graph = out(), torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    calls(first)
graph.replay()
second = out()
calls(second)
torch.cuda.synchronize()
assert all(bool(u.any()) and torch.equal(u, v) for u, v in zip(first, second))
print("equal")
"""


def test_first_calls_in_a_capture():
    p = subprocess.run([sys.executable, "-c", PROGRAM], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and "equal" in p.stdout, p.stderr[-2000:]

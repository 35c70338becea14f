"""Low-rank adapters (rwkvq_lowrank): the first call of a process is cut as all later ones are, and has their bits."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CALLS = """
import sys, torch
from paper_2505_03803_b200 import binding as B
T, rows, graph_first = (int(v) for v in sys.argv[1:])
g = torch.Generator(device="cuda").manual_seed(1)
x = torch.randn((T, 4096), generator=g, device="cuda").bfloat16()
A = (torch.randn((2, 64, 4096), generator=g, device="cuda") / 64).bfloat16()
Bm = torch.randn((2, 4096, 64), generator=g, device="cuda").bfloat16()
y0 = torch.randn((T, 4096), generator=g, device="cuda")
adapter = torch.zeros(T if rows else 1, dtype=torch.int32, device="cuda")
ys = [y0.clone() for _ in range(3)]
if graph_first:
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.rwkvq_lowrank(x, A, Bm, ys[0], adapter)
    graph.replay()
for y in ys[graph_first:]:
    B.rwkvq_lowrank(x, A, Bm, y, adapter)
torch.cuda.synchronize()
assert B.rwkvq_device_status() == 0
assert not torch.equal(ys[0], y0) and torch.equal(ys[0], ys[1]) and torch.equal(ys[1], ys[2]), (ys[0] - ys[1]).abs().max().item()
"""


# tiles, just as many as there are clusters of some width at once: fourteen and 57 of sixteen rows, 32 of 64; groups of rows, fifteen
@pytest.mark.parametrize("T,rows,graph_first", [(220, 0, 0), (900, 0, 0), (2048, 0, 0), (2048, 0, 1), (208, 1, 0)])
def test_the_first_call_has_the_bits_of_the_others(T, rows, graph_first):
    done = subprocess.run([sys.executable, "-c", CALLS, str(T), str(rows), str(graph_first)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]

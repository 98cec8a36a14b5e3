"""nuna_init in a process that has captured a graph and used a second stream before: workgroup 0 need no longer run on XCD
0 there, and XCD placement has to be available all the same.  The process is a child, so that nothing the other tests did
comes before, and nothing it does stays."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import torch
from paper_2608_00867_amd import nuna
y = torch.zeros(100, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    y.add_(1)
graph.replay()
with torch.cuda.stream(torch.cuda.Stream()):
    y.mul_(2)
torch.cuda.synchronize()
nuna.init()
assert nuna.device_info()["map_verified"] == 1
xcc, _ = nuna.probe_xcc(4096)
torch.cuda.synchronize()
b = torch.arange(4096, device="cuda")
assert bool(((xcc - xcc[0]) % 8 == b % 8).all()), "not a turned map"
ins = [torch.full((1 << 16,), float(r), device="cuda") for r in range(8)]
for placement in ("xcd", "linear"):
    for out in nuna.allreduce(ins, placement=placement):
        assert bool((out == 28).all())
print("first workgroup on XCD", int(xcc[0]))
"""


def test_init_after_a_graph_and_a_second_stream():
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT), capture_output=True,
                       text=True, timeout=110)
    assert r.returncode == 0, r.stdout[-1000:] + r.stderr[-3000:]
    print(r.stdout)

"""How many CTAs a call gets depends on its own sizes, not on the calls before it."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

PROGRAM = """
import json, sys, tempfile, torch
sys.path.insert(0, {root!r})
import paper_2508_02322_b200 as P

def step(rows, vocab):
    z = torch.randn(rows, vocab, device="cuda:0")
    idx = torch.arange(8, device="cuda:0", dtype=torch.int32).expand(rows, -1).contiguous()
    lp = torch.full((rows, 8), -3.0, device="cuda:0")
    P.camera_distill_step(z, idx, lp, torch.ones(rows, device="cuda:0"), tail=True)
    torch.cuda.synchronize()

for rows, vocab in {before}:
    step(rows, vocab)
from torch.profiler import profile, ProfilerActivity
with profile(activities=[ProfilerActivity.CUDA]) as p:
    step(400, 60000)
with tempfile.NamedTemporaryFile(suffix=".json") as f:
    p.export_chrome_trace(f.name)
    events = json.load(open(f.name))["traceEvents"]
print("GRID", [e["args"]["grid"] for e in events if "k_distill" in e.get("name", "") and "grid" in e.get("args", {{}})])
"""


def grid(before):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", PROGRAM.format(root=root, before=before)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr[-2000:]
    line = [l for l in out.stdout.splitlines() if l.startswith("GRID")]
    assert line and "[" in line[0][6:], out.stdout[-500:]
    return line[0]


def test_grid_does_not_depend_on_earlier_calls():
    fresh = grid([])
    # a vocabulary so long that one CTA fits an SM; the same kernel and split
    assert grid([(200, 1 << 20)]) == fresh
    assert grid([(200, 1 << 20), (400, 60000), (200, 1 << 20)]) == fresh

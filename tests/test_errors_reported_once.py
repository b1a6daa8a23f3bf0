"""An error of the CUDA runtime is reported by the call that met it, and by no later one."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import torch
import paper_2409_10644_b200 as m
dev = "cuda"
ws = m.new_workspace(1 << 20, dev)
x, rows = torch.randn(1, 3, 96, device=dev), torch.zeros(1, 3, 96, device=dev)
lens, freqs = torch.zeros(1, dtype=torch.int32, device=dev), torch.rand(16, dtype=torch.float64, device=dev)
torch.cuda.synchronize()
graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
failed = 0
with torch.cuda.stream(side):
    graph.capture_begin()
    failed = m.lib.mcsd_workspace_status(ws.data_ptr(), side.cuda_stream)     # synchronises, which a capture does not allow
    try:
        graph.capture_end()
    except Exception:
        pass
print("status", failed)
m.mcsd_latent_rows(x, None, lens, freqs, rows=rows)
torch.cuda.synchronize()
print("rows", bool((rows != 0).any()))
"""


@pytest.mark.gpu
def test_a_refused_synchronisation_is_not_reported_by_the_next_launch():
    r = subprocess.run([sys.executable, "-c", SCRIPT], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert "status -6" in r.stdout and "rows True" in r.stdout, r.stdout + r.stderr

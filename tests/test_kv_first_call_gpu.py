"""The first calls of a process may be captured ones."""
import os
import subprocess
import sys

import pytest

from paper_2608_24658_gb300 import build

pytestmark = pytest.mark.gpu

SCRIPT = """
import torch
from paper_2608_24658_gb300.api import kv_read, kv_scales, kv_write
k = torch.randn((40, 2, 128), device="cuda").bfloat16()
v = torch.randn((40, 2, 128), device="cuda").bfloat16()
pools = [torch.zeros((3, 2, 16, 128), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
slots = torch.arange(40, dtype=torch.int32, device="cuda")
ks, vs = torch.ones(2, device="cuda"), torch.ones(2, device="cuda")
rows = [torch.zeros_like(k) for _ in range(2)]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    kv_scales(k, v, k_scale=ks, v_scale=vs)
    kv_write(k, v, *pools, slots, k_scale=ks, v_scale=vs)
    kv_read(*pools, slots, k=rows[0], v=rows[1], k_scale=ks, v_scale=vs)
graph.replay()
torch.cuda.synchronize()
for got, want in zip(rows, (k, v)):
    # half a step of e4m3 and of bf16, half of the least step of e4m3 at the scale
    bound = want.float().abs() * (2.0 ** -4 + 2.0 ** -7) + 2.0 ** -10 * want.float().abs().amax() / 448
    assert ((got.float() - want.float()).abs() <= bound).all()
print("captured")
"""


def test_first_calls_are_captured():
    build.build()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", SCRIPT], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "captured" in done.stdout, done.stdout + done.stderr

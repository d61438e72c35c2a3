"""A process whose first calls of include/spec_ops.h are made under stream capture."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

CHILD = """
import torch
import paper_2504_00030_amd as pk
torch.manual_seed(0)
f8 = torch.float8_e4m3fn
cases = []
for R, N, K in ((1, 512, 1024), (9, 6000, 1040), (70, 8300, 400), (260, 6200, 400)):
    x = torch.randn((R, K), device="cuda").to(torch.bfloat16)
    w = torch.randn((N, K), device="cuda").to(f8)
    ws = torch.rand(((N + 127) // 128, (K + 127) // 128), device="cuda")
    work = torch.empty(132 * R * ((K + 127) // 128) + (32 << 20), dtype=torch.uint8, device="cuda")
    cases.append((x, w, ws, work, [torch.zeros((R, N), dtype=t, device="cuda") for t in (torch.float32, torch.bfloat16)],
                  torch.zeros((R, K), dtype=f8, device="cuda"), torch.zeros(((K + 127) // 128, R), device="cuda")))
h = torch.randn((5, 3, 128), device="cuda")
g, c = torch.ones(128, device="cuda"), torch.rand((8, 64), device="cuda")
pos = torch.tensor([0, 7, 3, -1, 2], dtype=torch.int32, device="cuda")
heads = torch.zeros_like(h)
torch.cuda.synchronize()

def run():
    s = torch.cuda.current_stream().cuda_stream
    for x, w, ws, work, ys, q, scale in cases:
        pk.k_quant_f8(x, q, scale, stream=s)
        for y in ys:
            pk.k_gemm_f8(w, ws, x, y, workspace=work, stream=s)
    pk.k_qk_norm_rope(h[:, :2], h[:, 2:], g, g, c, c, pos, heads[:, :2], heads[:, 2:], stream=s)

outs = [t for case in cases for t in (*case[4], case[5].view(torch.uint8), case[6])] + [heads]
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    run()
for t in outs:
    assert not t.any(), "a captured call ran"
run()
torch.cuda.synchronize()
want = [t.clone() for t in outs]
for i in range(3):
    for t in outs:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for t, u in zip(outs, want):
        assert t.any() and torch.equal(t, u)
    torch.randn(1 << 18, device="cuda").sum().item()
print("captured first")
"""


def test_first_calls_under_capture():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, PYTHONPATH=root)
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=root, env=env, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "captured first" in r.stdout, r.stdout + r.stderr

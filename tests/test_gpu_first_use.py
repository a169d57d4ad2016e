"""The operators' first call in a process, which prepares their kernels: made while a graph is captured, and by several threads at once."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SETUP = """
import threading
import torch
from paper_2511_11446_b200 import binding as B
n, H, D, C = 300, 4, 64, 256
g = torch.Generator(device="cuda").manual_seed(1)
x = torch.randn(n, 3 * C, generator=g, device="cuda").to(torch.bfloat16)
q, k, v = x.split(C, 1)
ws = torch.empty(B.dp_group_norm_workspace(1, n, C, 8), dtype=torch.uint8, device="cuda")
def call(y, z):
    B.dp_attention(B.make_attn(H, H, D, 1, n, n, 0.125), q, 3 * C, n, k, 3 * C, v, 3 * C, n, y, C)
    B.dp_group_norm(x, 1, n, C, 3 * C, 8, None, None, 1e-5, B.DP_ACT_SILU, z, C, ws)
out = lambda: [torch.zeros(n, C, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
torch.cuda.synchronize()
"""
CAPTURED = """
a, b = out(), out()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    call(*a)
graph.replay()
torch.cuda.synchronize()
call(*b)
torch.cuda.synchronize()
assert all(torch.equal(s, t) and s.any() for s, t in zip(a, b))
print("same")
"""
THREADS = """
outs = [out() for _ in range(6)]
go = threading.Barrier(6)
def work(y):
    go.wait()
    B.dp_attention(B.make_attn(H, H, D, 1, n, n, 0.125), q, 3 * C, n, k, 3 * C, v, 3 * C, n, y, C)
ts = [threading.Thread(target=work, args=(o[0],)) for o in outs]
[t.start() for t in ts]
[t.join() for t in ts]
torch.cuda.synchronize()
assert all(torch.equal(o[0], outs[0][0]) and o[0].any() for o in outs)
print("same")
"""


LINEAR = """
w = torch.randint(-127, 128, (256, 256), generator=torch.Generator().manual_seed(1), dtype=torch.int8)
packed = torch.from_numpy(B.dp_pack_weights_host(w.numpy(), 8)).cuda()
s_w, s_a, codes = torch.full((256,), 0.01, device="cuda"), torch.ones(n, device="cuda"), torch.randint(-127, 128, (n, 256), device="cuda").to(torch.int8)
wt = B.make_weight(packed, s_w, None, 256, 256, 8)
outs = [torch.zeros(n, 256, dtype=torch.bfloat16, device="cuda") for _ in range(6)]
torch.cuda.synchronize()
ts = [threading.Thread(target=lambda y=y: B.dp_wq_linear(wt, codes, 256, s_a, n, y, 256, None)) for y in outs]
[t.start() for t in ts]
[t.join() for t in ts]
torch.cuda.synchronize()
assert all(torch.equal(o, outs[0]) and o.any() for o in outs)
print("same")
"""


@pytest.mark.parametrize("body", [CAPTURED, THREADS, LINEAR], ids=["captured", "threads", "linear"])
def test_first_call(body):
    r = subprocess.run([sys.executable, "-c", SETUP + body], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]

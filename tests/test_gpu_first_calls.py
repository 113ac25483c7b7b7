"""A fresh process: the first context is made without loading the expert and norm kernels, and their first call may be a captured one."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import json, time, torch
torch.zeros(1 << 20, device="cuda").sum().item()
from paper_2508_12801_b200 import binding as ms
t0 = time.perf_counter()
ctx = ms.create(ms.make_params(64, 256, 8, 2, 1.0, io_dtype=ms.BF16), "cuda:0")
create_ms = (time.perf_counter() - t0) * 1e3
C, bf = ctx.capacity, dict(dtype=torch.bfloat16, device="cuda:0")
x, w, y = torch.randn(8, C, 256, **bf), torch.randn(8, 256, 512, **bf), torch.zeros(8, C, 512, **bf)
load = torch.full((8,), C, dtype=torch.int32, device="cuda:0")
wide = ms.create(ms.make_params(300, 256, 8, 1, capacity=300, io_dtype=ms.BF16), "cuda:0")
X, Y, L = torch.randn(8, 300, 256, **bf), torch.zeros(8, 300, 512, **bf), torch.full((8,), 300, dtype=torch.int32, device="cuda:0")
dw = torch.zeros(8, 256, 512, device="cuda:0")
r, wn = torch.randn(64, 256, **bf), torch.ones(256, **bf)
h, dr, dpre, n = torch.zeros_like(r), torch.zeros_like(r), torch.zeros(256, device="cuda:0"), ms.make_norm(w_pre=wn)
def calls():
    ms.expert_gemm(ctx, x, w, load, y, 256, 512)
    ms.expert_gemm(wide, X, w, L, Y, 256, 512)
    ms.expert_gemm_dw(wide, X, Y, L, dw, 256, 512)
    ms.block_norm(ctx, None, r, n, None, h)
    ms.block_norm_bwd(ctx, None, h, None, r, n, None, dr, None, None, dpre)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (y, Y, dw, h, dr, dpre)]
for t in (y, Y, dw, h, dr, dpre):
    t.fill_(float("nan"))
calls()
torch.cuda.synchronize()
same = all(torch.equal(a, b) and bool(a.abs().max() > 0) for a, b in zip(got, (y, Y, dw, h, dr, dpre)))
print(json.dumps(dict(create_ms=create_ms, same=same, flags=ms.check_internal(ctx) | ms.check_internal(wide))))
"""


def test_first_context_and_first_captured_calls():
    best = float("inf")
    for _ in range(3):                       # the first start on a machine also reads the files
        p = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, capture_output=True, text=True, timeout=300)
        assert p.returncode == 0, p.stderr[-2000:]
        r = json.loads(p.stdout.strip().splitlines()[-1])
        assert r["same"] and r["flags"] == 0
        best = min(best, r["create_ms"])
        if best < 25:
            break
    assert best < 25, f"the first context took {best:.1f} ms (7 ms where only the router's kernels are loaded, 48 ms with all of them)"

"""A fresh process whose first calls of top-k routing and of the 8-bit forms are captured ones."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import json, torch
from paper_2508_12801_b200 import binding as ms
from paper_2508_12801_b200.layer import MoELayer
g = torch.Generator().manual_seed(1)
r = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).to(torch.bfloat16).to("cuda:0")
def make(T, d, E, k, f):                  # few rows an expert, and many
    p, how = ms.make_params(T, d, E, k, 1.5, io_dtype=ms.BF16), ms.make_topk(ms.SIGMOID, 4, 2, True)
    train, serve = MoELayer(p, f, topk=how, keep8=True), MoELayer(p, f, topk=how, training=False, int8=True)
    h, res, wg, wu, wd, dro, dho = r(T, d), r(T, d), r(d, E, scale=d ** -0.5), r(E, d, 2 * f, scale=d ** -0.5), r(E, f, d, scale=f ** -0.5), r(T, d), r(T, d)
    norm, bias = ms.make_norm(w_pre=r(d)), torch.zeros(E, device="cuda:0")
    out = [torch.zeros_like(res) for _ in range(6)] + [torch.zeros(*t.shape, device="cuda:0") for t in (wg, wu, wd)] + [torch.zeros(d, device="cuda:0")]
    q = [(torch.zeros(E, n, m, dtype=torch.int8, device="cuda:0"), torch.zeros(E, n, device="cuda:0")) for n, m in ((2 * f, d), (d, f))]
    def calls():
        train.forward(h, res, wg, wu, wd, norm, out[0], out[1], balance_bias=bias)
        train.backward(dro, dho, h, out[0], wg, wu, wd, norm, out[2], out[3], *out[6:9], dw_pre=out[9])
        ms.expert_quant_weight(serve.ctx, wu, *q[0], d, 2 * f)
        ms.expert_quant_weight(serve.ctx, wd, *q[1], f, d)
        serve.forward(h, res, wg, *q, norm, out[4], out[5], balance_bias=bias)
    return calls, out, (train.ctx, serve.ctx)
sets = [make(40, 128, 8, 2, 64), make(3000, 128, 8, 2, 64)]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    for calls, _, _ in sets:
        calls()
graph.replay()
torch.cuda.synchronize()
outs = [t for _, out, _ in sets for t in out]
got = [t.clone() for t in outs]
for t in outs:
    t.fill_(float("nan"))
for calls, _, _ in sets:
    calls()
torch.cuda.synchronize()
same = [torch.allclose(a, b, rtol=1e-4, atol=1e-4) if a.dtype == torch.float32 else torch.equal(a, b) for a, b in zip(got, outs)]
print(json.dumps(dict(same=all(same), some=all(bool(a.abs().max() > 0) for a in got), flags=sum(ms.check_internal(c) for _, _, cs in sets for c in cs))))
"""


def test_first_calls_are_captured():
    p = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr[-2000:]
    assert json.loads(p.stdout.strip().splitlines()[-1]) == dict(same=True, some=True, flags=0)

"""Operators on device tensors whose first call of all is captured into a graph, in a process of its own."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import torch
import paper_2510_23264_amd as P
g = torch.Generator(device="cuda").manual_seed(5)
def held(rows, k):
    return P.Mx4(torch.randint(0, 256, (rows, k // 2), generator=g, device="cuda", dtype=torch.uint8),
                 torch.randint(118, 126, (rows, k // 32), generator=g, device="cuda", dtype=torch.uint8), k)
# the kernel of few rows and the five forms of tiles (tests/mx4_rules.py)
pairs = [(held(m, k), held(n, k)) for m, n, k in ((3, 200, 512), (40, 60, 512), (33, 8681, 1536), (65, 8308, 1536), (257, 7834, 1536), (1410, 8141, 1536))]
x, t, pos = torch.randn(50, 6, 64, device="cuda"), P.rotary_table(32), torch.arange(50, device="cuda")
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    q = P.mx4_quantize(x.view(50, 384))
    down = P.mx4_quantize(x.view(50, 384), by="columns")
    values = P.mx4_dequantize(q)
    turned = P.rotary(x, pos, t)
    products = [P.mx4_gemm(a, w, dtype=torch.bfloat16) for a, w in pairs]
for _ in range(4):
    x.normal_()
    for a, w in pairs:
        a.codes.random_(0, 256, generator=g)
    graph.replay()
    torch.cuda.synchronize()
    again = P.mx4_quantize(x.view(50, 384))
    assert torch.equal(q.codes, again.codes) and torch.equal(q.scales, again.scales)
    assert torch.equal(down.codes, P.mx4_quantize(x.view(50, 384), by="columns").codes)
    assert torch.equal(values, P.mx4_dequantize(again)) and torch.equal(turned, P.rotary(x, pos, t))
    assert all(torch.equal(y, P.mx4_gemm(a, w, dtype=torch.bfloat16)) for y, (a, w) in zip(products, pairs))
    torch.cuda.synchronize()
print("replayed")
"""


def test_the_first_call_is_a_captured_one():
    got = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=100)
    assert got.returncode == 0 and "replayed" in got.stdout, got.stdout

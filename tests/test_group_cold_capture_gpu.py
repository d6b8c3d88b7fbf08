"""Grouped layers, their gradient and updates captured into a graph by the first call that a
process makes of them: what is set up once is set up without disturbing the capture."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

PROGRAM = """
import sys
import torch
from paper_2609_09020_gb300 import pic
kind, dtype, rows, K, N = sys.argv[1], getattr(torch, sys.argv[2]), *map(int, sys.argv[3:])
g = torch.Generator(device="cuda").manual_seed(0)
normal = lambda *s: torch.randn(s, generator=g, device="cuda").mul_(0.1).to(dtype)
x, w, b, dy = normal(rows, K), normal(3, N, K), normal(3, N), normal(rows, N)
o = torch.tensor([0, rows // 3, rows // 3, rows], device="cuda")
m = [normal(N, K), normal(64, 64)]
out = [torch.zeros_like(t) for t in m]
h = pic.Orthogonalizer(m, out=out)
calls = {"forward": lambda: [pic.grouped_linear(x, w, o, b, act="gelu")],
         "backward": lambda: list(pic.grouped_linear_backward(dy, x, w, o, act="none")),
         "orth": lambda: h.orthogonalize() or out}
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    held = calls[kind]()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in held]
want = calls[kind]()
pic.grouped_linear_check()
h.check()
assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(bool(t.any()) for t in got)
print("same")
"""


@pytest.mark.parametrize("kind", ["forward", "backward", "orth"])
@pytest.mark.parametrize("dtype,rows,K,N", [("float16", 3000, 64, 64), ("bfloat16", 1000, 264, 200), ("float32", 4000, 256, 512),
                                            ("float32", 20, 520, 264), ("float16", 500, 333, 517)])
def test_first_call_captured(kind, dtype, rows, K, N):
    from paper_2609_09020_gb300 import build
    build.build()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", PROGRAM, kind, dtype, str(rows), str(K), str(N)], cwd=root, timeout=120,
                       capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]

"""Dense operators captured by a process that has made no call of theirs before, with results that are finite and exact: every sum counts."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

CODE = """
import torch
from paper_2011_05630_b200 import dense
gen = torch.Generator(device="cuda").manual_seed(0)
whole = lambda *s: torch.randint(-1, 2, s, generator=gen, device="cuda").half()
M = %d
x, w, wu, dy, z = whole(M, 520), whole(264, 520), whole(264, 520), whole(M, 264), whole(M, 264)
torch.cuda.synchronize()


def calls():
    return [dense.linear(x, w, residual=dy), *dense.gated(x, w, wu, act="relu", save=True), *dense.linear_backward(dy, x, w, z, act="relu", residual=True),
            *dense.linear_backward(dy, x, w)[:3], *dense.gated_backward(dy, x, w, wu, z, dy, act="relu", bias=True)]


g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    got = calls()
for t in got:
    t.fill_(float("nan"))
X, W, U, E, Z = (t.double() for t in (x, w, wu, dy, z))
G, V, D = X @ W.t(), X @ U.t(), E * (Z > 0)
dg, du = E * E * (Z > 0), E * Z.relu()
want = [G + E, G.relu() * V, G, V, D @ W, D.t() @ X, D.sum(0), D, E @ W, E.t() @ X, E.sum(0), dg @ W + du @ U, dg.t() @ X, du.t() @ X, dg.sum(0), du.sum(0)]
assert len(want) == len(got)
for again in range(2):
    g.replay()
    dense.synchronize()
    for i, (p, q) in enumerate(zip(got, want)):
        assert float(q.abs().max()) < 60000
        assert torch.equal(p, q.to(p.dtype)), i
    x.copy_(whole(M, 520))   # (a replay reads what lies there then)
    X = x.double()
    G, V = X @ W.t(), X @ U.t()
    want = [G + E, G.relu() * V, G, V, D @ W, D.t() @ X, D.sum(0), D, E @ W, E.t() @ X, E.sum(0), dg @ W + du @ U, dg.t() @ X, du.t() @ X, dg.sum(0), du.sum(0)]
print("captured")
"""


@pytest.mark.parametrize("m", [3, 40, 300, 1500])
def test_captured_before_any_other_call(m):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CODE % m], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]

"""Which kernels dense operators launched, asked from Python and printed by the command line."""
import os
import subprocess
import sys
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2011_05630_b200 import dense
from tests.test_gpu_dense import Maker


def test_kernels_of_a_call():
    mk = Maker(1, torch.float16)
    x, w, y = mk.mat(300, 128), mk.mat(72, 128), mk.mat(300, 72)
    assert [t.split("(")[0] for t in dense.kernels(lambda: (dense.linear(x[:3], w), dense.linear(x, w)))] == ["dense_gemv", "dense_lat"]
    other = []

    def call():   # another thread's calls are another's business
        t = threading.Thread(target=lambda: other.append(dense.linear(x, w)))
        t.start()
        t.join()
        dense.linear_backward(y, x, w, y, act="relu")

    (text,) = dense.kernels(call)
    assert text.startswith("dense_grad(") and "; dense_lat(" in text and torch.equal(other[0], dense.linear(x, w))
    with pytest.raises(ValueError):
        dense.kernels(lambda: dense.linear(x, y))
    assert dense.kernels(lambda: None) == []


@pytest.mark.parametrize("op,flags", [("linear", ["--residual", "--act", "gelu"]), ("gated", [])])
def test_the_command_line(op, flags):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-m", "paper_2011_05630_b200.layer_cli", "2", "7", "5", "136", "200", "1", "--op", op, "--dtype", "bf16", "--backward", *flags],
                       cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = r.stdout.splitlines()
    assert lines[0].startswith("%s forward, 70 tokens of 136 -> 200, bf16" % op) and lines[1].strip().startswith("dense_lat(")
    assert lines[2].startswith("%s backward" % op) and lines[3].strip().startswith("dense_grad(")

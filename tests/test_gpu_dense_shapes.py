"""Tensors that are no matrices are refused as such, whichever of a call's they are."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2011_05630_b200 import dense
from tests.test_gpu_dense import Maker


def test_matrices_of_another_number_of_dimensions_are_refused():
    mk = Maker(2, torch.float16)
    x, w, y = mk.mat(5, 64), mk.mat(40, 64), mk.mat(5, 40)
    for f in (lambda: dense.linear(x, w[0, 0]), lambda: dense.linear(x, w[0]), lambda: dense.linear(x, w[None]), lambda: dense.linear(x, w, residual=y[0]),
              lambda: dense.linear_backward(y, x[0], w), lambda: dense.linear_backward(y, x[0, 0], w), lambda: dense.linear_backward(y, x, w[0]),
              lambda: dense.linear_backward(y, None, w[0], need_dw=False), lambda: dense.linear_backward(y, x, None, y[0], act="silu", need_dx=False),
              lambda: dense.gated(x, w[0, 0], w), lambda: dense.gated(x, w, w[0]), lambda: dense.gated_backward(y, x[0], w, w, y, y),
              lambda: dense.gated_backward(y, None, w[0], w, y, y, need_dw=False), lambda: dense.gated_backward(y, x, w, w, y, y[0])):
        with pytest.raises(ValueError):
            f()

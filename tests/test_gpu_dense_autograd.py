"""The dense operators record nothing for autograd: where it would have recorded, a tensor that requires a gradient is refused."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2011_05630_b200 import dense
from tests.test_gpu_dense import Maker

CALLS = {
    "linear": lambda t: dense.linear(t["x"], t["w"], t["b"], t["y"], act="gelu", out=t["out"]),
    "linear_backward": lambda t: dense.linear_backward(t["y"], t["x"], t["w"], t["z"], act="gelu"),
    "gated": lambda t: dense.gated(t["x"], t["w"], t["wu"], t["b"], t["bu"], out=t["out"]),
    "gated_backward": lambda t: dense.gated_backward(t["y"], t["x"], t["w"], t["wu"], t["z"], t["out"]),
}
USED = {"linear": "x w b y out", "linear_backward": "y x w z", "gated": "x w wu b bu out", "gated_backward": "y x w wu z out"}


def tensors():
    mk = Maker(2, torch.bfloat16)
    return {"x": mk.mat(5, 64), "w": mk.mat(40, 64), "wu": mk.mat(40, 64), "y": mk.mat(5, 40), "z": mk.mat(5, 40), "out": mk.mat(5, 40), "b": mk.vec(40), "bu": mk.vec(40)}


@pytest.mark.parametrize("op,name", [(op, name) for op in CALLS for name in USED[op].split()])
def test_what_autograd_would_lose_is_refused(op, name):
    t = tensors()
    CALLS[op](t)
    t[name].requires_grad_(True)
    before = t["out"].detach().clone()
    with pytest.raises(ValueError, match="gradient"):
        CALLS[op](t)
    assert torch.equal(t["out"].detach(), before)
    with torch.no_grad():
        CALLS[op](t)
    t[name] = t[name].detach()
    CALLS[op](t)

"""Dense operators called from host threads that have made no other call of CUDA's: the first one may be any of them, and in a training loop's
backward pass it is."""
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2011_05630_b200 import dense
from tests import dense_util as D
from tests.test_gpu_dense import Maker


def in_a_new_thread(f):
    out = []

    def run():
        try:
            out.append(f())
        except Exception as e:
            out.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    if isinstance(out[0], Exception):
        raise out[0]
    return out[0]


@pytest.mark.parametrize("size", [(3, 256, 130), (40, 320, 712), (130, 200, 333), (1030, 192, 2056)], ids=str)
def test_the_first_call_of_a_thread(size):
    m, k, n = size
    mk = Maker(sum(size), torch.bfloat16)
    x, w, wu, dy, z, u = mk.mat(m, k), mk.mat(n, k, k ** -0.5), mk.mat(n, k, k ** -0.5), mk.mat(m, n), mk.mat(m, n), mk.mat(m, n)
    for f in (lambda: [dense.linear(x, w, residual=dy)], lambda: [dense.gated(x, w, wu)], lambda: dense.linear_backward(dy, x, w, z, act="silu"),
              lambda: dense.linear_backward(dy, x, w), lambda: dense.gated_backward(dy, x, w, wu, z, u, bias=True)):
        want = f()
        f()   # (the allocator has memory for the results: no call of the runtime's in the new thread but the operator's)
        torch.cuda.synchronize()
        got = in_a_new_thread(f)
        assert all(torch.equal(p, q) for p, q in zip(got, want) if p is not None)
    in_a_new_thread(dense.synchronize)


def test_an_autograd_function_of_a_block():
    """A gated block with its way back as a Function: its gradients reach leaves by autograd and are the operators' own."""

    class Block(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, wg, wu, wd):
            h, g, u = dense.gated(x, wg, wu, save=True)
            ctx.save_for_backward(x, wg, wu, wd, h, g, u)
            return dense.linear(h, wd, residual=x)

        @staticmethod
        def backward(ctx, dy):
            x, wg, wu, wd, h, g, u = ctx.saved_tensors
            dh, dwd, _, dr = dense.linear_backward(dy, h, wd, bias=False, residual=True)
            dx, dwg, dwu, _, _ = dense.gated_backward(dh, x, wg, wu, g, u)
            return dx + dr, dwg, dwu, dwd

    mk = Maker(3, torch.float16)
    m, k, n = 48, 128, 320
    leaves = [mk.mat(m, k), mk.mat(n, k, k ** -0.5), mk.mat(n, k, k ** -0.5), mk.mat(k, n, n ** -0.5)]
    dy = mk.mat(m, k)
    for t in leaves:
        t.requires_grad_(True)
    Block.apply(*leaves).backward(dy)
    doubles = [t.detach().double().requires_grad_(True) for t in leaves]
    x, wg, wu, wd = doubles
    (D.act(x @ wg.t(), "silu") * (x @ wu.t()) @ wd.t() + x).backward(dy.double())
    for got, want in zip(leaves, doubles):   # (five roundings to fp16 on the way, each off by half a step at most: 2^-11 of the value)
        assert float((got.grad.double() - want.grad).norm()) <= 5 * 2.0 ** -11 * float(want.grad.norm())

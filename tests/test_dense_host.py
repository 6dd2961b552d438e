"""What the dense operators refuse, decided on the host from the arguments alone (the pointers are dummies: no device call is made), and
the workspace that they ask for."""
import ctypes as C

import pytest

from paper_2011_05630_b200 import binding as B, dense as D

P = 1 << 20   # a dummy pointer


def linear(**kw):
    a = dict(dtype=1, act=0, m=4, k=64, n=32, x=P, w=2 * P, bias=0, res=0, y=3 * P, z=0, ldx=64, ldw=64, ldres=32, ldy=32, ldz=32)
    a.update(kw)
    return "dlf_linear", D._LINEAR.pack(*a.values())


def linear_grad(**kw):
    a = dict(dtype=0, act=3, m=4, k=64, n=32, dy=P, x=2 * P, w=3 * P, z=4 * P, dx=5 * P, dw=6 * P, db=7 * P, dz=0,
             lddy=32, ldx=64, ldw=64, ldz=32, lddx=64, lddw=64, lddz=32)
    a.update(kw)
    return "dlf_linear_grad", D._LINEAR_GRAD.pack(*a.values())


def gated(**kw):
    a = dict(dtype=1, act=5, m=4, k=64, n=32, x=P, wg=2 * P, wu=3 * P, bg=0, bu=0, h=4 * P, g=0, u=0, ldx=64, ldwg=64, ldwu=64, ldh=32, ldg=32, ldu=32)
    a.update(kw)
    return "dlf_gated", D._GATED.pack(*a.values())


def gated_grad(**kw):
    a = dict(dtype=1, act=5, m=4, k=64, n=32, dh=P, x=2 * P, wg=3 * P, wu=4 * P, g=5 * P, u=6 * P, dx=7 * P, dwg=8 * P, dwu=9 * P, dbg=0, dbu=0,
             lddh=32, ldx=64, ldwg=64, ldwu=64, ldg=32, ldu=32, lddx=64, lddwg=64, lddwu=64)
    a.update(kw)
    return "dlf_gated_grad", D._GATED_GRAD.pack(*a.values())


@pytest.mark.parametrize("make", [linear, linear_grad, gated, gated_grad])
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), B.E_INVALID_ARG), (dict(dtype=-1), B.E_INVALID_ARG), (dict(act=6), B.E_INVALID_ARG), (dict(act=-1), B.E_INVALID_ARG),
    (dict(m=-1), B.E_SHAPE), (dict(k=0), B.E_SHAPE), (dict(n=0), B.E_SHAPE), (dict(n=(1 << 30) + 1), B.E_SHAPE), (dict(m=1 << 40), B.E_SHAPE),
    (dict(ldx=63), B.E_SHAPE), (dict(ldx=-64), B.E_SHAPE), (dict(ldx=1 << 40), B.E_SHAPE), (dict(x=0), B.E_INVALID_ARG), (dict(x=P + 1), B.E_INVALID_ARG)])
def test_refusals_that_all_share(make, kw, status):
    op, args = make(**kw)
    need = C.c_size_t(7)
    assert getattr(B.lib(), op)(args, 4096, 1 << 40, None) == status
    assert getattr(B.lib(), op + "_workspace_bytes")(args, C.byref(need)) == status


@pytest.mark.parametrize("make,kw,status", [
    (linear, dict(w=0), B.E_INVALID_ARG), (linear, dict(y=0), B.E_INVALID_ARG), (linear, dict(bias=P + 2), B.E_INVALID_ARG),
    (linear, dict(res=P, ldres=31), B.E_SHAPE), (linear, dict(z=P, ldz=3), B.E_SHAPE), (linear, dict(ldw=63), B.E_SHAPE), (linear, dict(ldy=1), B.E_SHAPE),
    (linear_grad, dict(dy=0), B.E_INVALID_ARG), (linear_grad, dict(w=0), B.E_INVALID_ARG), (linear_grad, dict(z=0), B.E_INVALID_ARG),
    (linear_grad, dict(db=P + 2), B.E_INVALID_ARG), (linear_grad, dict(lddx=60), B.E_SHAPE), (linear_grad, dict(lddw=60), B.E_SHAPE),
    (gated, dict(wg=0), B.E_INVALID_ARG), (gated, dict(wu=0), B.E_INVALID_ARG), (gated, dict(h=0), B.E_INVALID_ARG), (gated, dict(ldwu=10), B.E_SHAPE),
    (gated, dict(bu=P + 1), B.E_INVALID_ARG), (gated, dict(u=P, ldu=1), B.E_SHAPE),
    (gated_grad, dict(dh=0), B.E_INVALID_ARG), (gated_grad, dict(g=0), B.E_INVALID_ARG), (gated_grad, dict(u=0), B.E_INVALID_ARG),
    (gated_grad, dict(wu=0), B.E_INVALID_ARG), (gated_grad, dict(dbg=P + 2), B.E_INVALID_ARG), (gated_grad, dict(lddwu=5), B.E_SHAPE)])
def test_refusals_of_one(make, kw, status):
    op, args = make(**kw)
    assert getattr(B.lib(), op)(args, 4096, 1 << 40, None) == status


@pytest.mark.parametrize("make,kw", [
    (linear, dict(y=P)), (linear, dict(z=2 * P)), (linear, dict(z=3 * P)), (linear, dict(res=3 * P, ldres=40)), (linear, dict(res=5 * P, z=5 * P)),
    (linear_grad, dict(dx=2 * P)), (linear_grad, dict(dw=3 * P)), (linear_grad, dict(dx=P)), (linear_grad, dict(dw=4 * P)), (linear_grad, dict(dz=5 * P)),
    (linear_grad, dict(dz=P, lddz=48)), (linear_grad, dict(dz=4 * P, lddz=48)), (linear_grad, dict(dz=2 * P)),
    (gated, dict(h=P)), (gated, dict(g=4 * P)), (gated, dict(u=2 * P)), (gated, dict(g=8 * P, u=8 * P)),
    (gated_grad, dict(dx=P)), (gated_grad, dict(dwg=9 * P)), (gated_grad, dict(dwu=4 * P)), (gated_grad, dict(dbg=7 * P)), (gated_grad, dict(dx=5 * P))])
def test_outputs_over_inputs_are_refused(make, kw):
    op, args = make(**kw)
    assert getattr(B.lib(), op)(args, 4096, 1 << 40, None) == B.E_INVALID_ARG


def test_null_arguments():
    for op in ("dlf_linear", "dlf_linear_grad", "dlf_gated", "dlf_gated_grad"):
        assert getattr(B.lib(), op)(None, None, 0, None) == B.E_INVALID_ARG
        assert getattr(B.lib(), op + "_workspace_bytes")(None, C.byref(C.c_size_t())) == B.E_INVALID_ARG
    assert B.lib().dlf_linear_workspace_bytes(linear()[1], None) == B.E_INVALID_ARG


def need(op_args):
    n = C.c_size_t(7)
    assert getattr(B.lib(), op_args[0] + "_workspace_bytes")(op_args[1], C.byref(n)) == B.OK
    return n.value


def test_workspace():
    assert need(linear()) == 0 and need(gated()) == 0             # nothing where rows start on 16-byte boundaries
    assert need(linear_grad()) == 512                             # dz: 4 rows of 32 values, 64 apart
    assert need(linear_grad(act=0, z=0)) == 0 and need(linear_grad(dz=8 * P)) == 0
    assert need(linear_grad(dx=0, dw=0)) == 0 and need(linear_grad(m=0)) == 0
    assert need(gated_grad()) == 1024 and need(gated_grad(dx=0, dwu=0)) == 512
    for op, args in (linear_grad(), gated_grad()):
        f = getattr(B.lib(), op)
        assert f(args, None, 1 << 20, None) == B.E_WORKSPACE and f(args, 4096, 511, None) == B.E_WORKSPACE and f(args, 4096 + 16, 1 << 20, None) == B.E_WORKSPACE


def test_tensors_off_the_device_are_refused():
    torch = pytest.importorskip("torch")
    t = torch.zeros((2, 8), dtype=torch.float16)
    for f in (lambda: D.linear(t, t), lambda: D.gated(t, t, t), lambda: D.linear_backward(t, t, t), lambda: D.gated_backward(t, t, t, t, t, t)):
        with pytest.raises(ValueError):
            f()

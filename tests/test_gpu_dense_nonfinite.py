"""Infinities and NaN on the way back through the dense operators: nothing comes through an activation that is closed (ReLU and ReLU6, as
autograd has it), and what comes through an open one stays in its row of dx and its column's row of dw."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2011_05630_b200 import dense
from tests.test_gpu_dense import Maker, TYPES, ids

INF, NAN = float("inf"), float("nan")
SIZES = [(1, 64, 40), (5, 72, 33), (40, 136, 200), (300, 100, 130), (1500, 64, 24)]   # whole and odd rows, wide and narrow strips


def closed(z, a):
    """Four places with z where `a` is closed, its corners among them; the values at which no gradient may come through."""
    m, n = z.shape
    at = [(0, 0), (m // 2, n // 3), (m - 1, n - 1), (m // 3, n // 2)]
    for (i, j), v in zip(at, (-1.0, 0.0, NAN, 7.0 if a == "relu6" else -INF)):
        z[i, j] = v
    return at


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("a", ["relu", "relu6"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_nothing_comes_through_a_closed_activation(size, a, dtype):
    m, k, n = size
    mk = Maker(sum(size), dtype)
    dy, x, w, z = mk.mat(m, n), mk.mat(m, k), mk.mat(n, k, k ** -0.5), mk.mat(m, n, 2.0)
    at = closed(z, a)
    want = dense.linear_backward(dy, x, w, z, act=a, residual=True)
    for bad in (INF, -INF, NAN):
        for i, j in at:
            dy[i, j] = bad
        got = dense.linear_backward(dy, x, w, z, act=a, residual=True)
        assert all(float(got[3][i, j]) == 0.0 for i, j in at)
        for name, p, q in zip(("dx", "dw", "db", "dr"), got, want):
            assert torch.equal(p, q), name
    dense.synchronize()


@pytest.mark.parametrize("a", ["relu", "relu6"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_a_gated_block_with_a_closed_gate(size, a):
    """dg is 0 there whatever dh and u are; du = dh act(g) is a product like any other: 0 with a finite dh, NaN with an infinite one."""
    m, k, n = size
    mk = Maker(sum(size) + 1, torch.bfloat16)
    dh, x, wg, wu, g, u = mk.mat(m, n), mk.mat(m, k), mk.mat(n, k, k ** -0.5), mk.mat(n, k, k ** -0.5), mk.mat(m, n, 2.0), mk.mat(m, n)
    at = closed(g, "relu")   # (ReLU6 from 6 on is closed and not 0)
    want = dense.gated_backward(dh, x, wg, wu, g, u, act=a, bias=True)
    for i, j in at:
        u[i, j] = INF
    for p, q in zip(dense.gated_backward(dh, x, wg, wu, g, u, act=a, bias=True), want):
        assert torch.equal(p, q)
    for i, j in at:
        dh[i, j], u[i, j] = INF, NAN
    dx, dwg, dwu, dbg, dbu = dense.gated_backward(dh, x, wg, wu, g, u, act=a, bias=True)
    assert torch.equal(dwg, want[1]) and torch.equal(dbg, want[3])
    rows, cols = {i for i, _ in at}, {j for _, j in at}
    assert all(bool(torch.isnan(dx[i]).all()) for i in rows) and all(bool(torch.isnan(dwu[j]).all()) for j in cols)
    keep, other = [i for i in range(m) if i not in rows], [j for j in range(n) if j not in cols]
    assert torch.equal(dx[keep], want[0][keep]) and torch.equal(dwu[other], want[2][other]) and torch.equal(dbu[other], want[4][other])


@pytest.mark.parametrize("a", ["none", "relu", "relu6", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradients_that_are_not_finite_stay_in_their_rows(size, a):
    m, k, n = size
    mk = Maker(sum(size) + 2, torch.float16)
    dy, x, w, z, u = mk.mat(m, n), mk.mat(m, k), mk.mat(n, k, k ** -0.5), mk.mat(m, n), mk.mat(m, n)
    i, j = m // 2, n // 2
    z[i, j] = 1.5   # open in all of them
    clean = dense.linear_backward(dy, x, w, z, act=a, residual=a != "none"), dense.gated_backward(dy, x, w, w, z, u, act=a, bias=True)
    dy[i, j] = NAN
    after = dense.linear_backward(dy, x, w, z, act=a, residual=a != "none"), dense.gated_backward(dy, x, w, w, z, u, act=a, bias=True)
    keep, other = [r for r in range(m) if r != i], [c for c in range(n) if c != j]
    for before, now in zip(clean, after):
        assert bool(torch.isnan(now[0][i]).all()) and torch.equal(now[0][keep], before[0][keep])
    (_, dw, db, dr), (_, dwg, dwu, dbg, dbu) = after
    for p, q in zip((dw, db, dwg, dwu, dbg, dbu), (*clean[0][1:3], *clean[1][1:])):
        assert bool(torch.isnan(p[j]).all()) and torch.equal(p[other], q[other])
    if dr is not None:
        assert bool(torch.isnan(dr[i, j])) and int(torch.isnan(dr).sum()) == 1

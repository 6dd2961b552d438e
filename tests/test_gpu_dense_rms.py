"""The dense operators' results are rounded as often as they say and no more: once, and dz, dg and du once before they enter the products."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2011_05630_b200 import dense
from tests import dense_bounds as R, dense_util as D
from tests.test_gpu_dense import Maker

# (Long sums in fp32 would hide a second rounding: up to these many terms they do not.)
MOST = {torch.float16: 128, torch.bfloat16: 900}
SIZES = [((300, 128, 100), torch.float16), ((128, 64, 128), torch.float16), ((16, 128, 520), torch.float16), ((100, 60, 51), torch.float16)]
SIZES += [(s, torch.bfloat16) for s in ((300, 128, 100), (16, 900, 520), (777, 600, 401), (64, 850, 640), (900, 888, 2048), (1500, 555, 1333))]
ids = lambda v: str(v).replace("torch.", "")


@pytest.mark.parametrize("size,dtype", SIZES, ids=ids)
def test_forward(size, dtype):
    m, k, n = size
    mk = Maker(sum(size), dtype)
    x, w, wu, r, b = mk.mat(m, k), mk.mat(n, k, k ** -0.5), mk.mat(n, k, k ** -0.5), mk.mat(m, n), mk.vec(n)
    xd, wd, ud = x.double(), w.double(), wu.double()
    absum = xd.abs() @ wd.abs().t() + r.double().abs() + b.double().abs()
    z = xd @ wd.t() + b.double() + r.double()
    for a in ("none", "gelu", "gelu_tanh", "silu"):
        y, kept = dense.linear(x, w, b, r, act=a, save=True)
        R.check_rms(kept, z, k, absum, "z")
        R.check_rms(y, D.act(z, a), k, D.LIP * absum, "y " + a)
    g, u = xd @ wd.t(), xd @ ud.t()
    h, gk, uk = dense.gated(x, w, wu, save=True)
    R.check_rms(gk, g, k, xd.abs() @ wd.abs().t(), "g")
    R.check_rms(uk, u, k, xd.abs() @ ud.abs().t(), "u")
    if k <= MOST[dtype] * 2 // 3:
        R.check_rms(h, D.act(g, "silu") * u, k, (xd.abs() @ wd.abs().t()) * u.abs() + D.act(g, "silu").abs() * (xd.abs() @ ud.abs().t()), "h")


@pytest.mark.parametrize("size,dtype", SIZES, ids=ids)
def test_backward(size, dtype):
    m, k, n = size
    mk = Maker(sum(size) + 1, dtype)
    dy, x, w, z, wu, u = mk.mat(m, n), mk.mat(m, k), mk.mat(n, k), mk.mat(m, n), mk.mat(n, k), mk.mat(m, n)
    xd, wd, ud = x.double(), w.double(), wu.double()

    def product(got, terms, what, *pairs):
        if terms > MOST[dtype]:
            return
        pairs = [(R.rounded(p, dtype), q) for p, q in pairs]
        R.check_rms(got, sum(p @ q for p, q in pairs), terms, sum(p.abs() @ q.abs() for p, q in pairs), what)

    for a in ("none", "gelu", "gelu_tanh", "silu"):
        d = dy.double() * D.act_grad(z.double(), a)
        dx, dw, _, dr = dense.linear_backward(dy, x, w, z, act=a, residual=True)
        product(dx, n, "dx " + a, (d, wd))
        product(dw, m, "dw " + a, (d.t(), xd))
        if a != "none":
            R.check_rms(dr, d, 0, torch.zeros(1), "dr " + a)
    dg, du = dy.double() * u.double() * D.act_grad(z.double(), "silu"), dy.double() * D.act(z.double(), "silu")
    dx, dwg, dwu, _, _ = dense.gated_backward(dy, x, w, wu, z, u)
    product(dx, 2 * n, "gated dx", (dg, wd), (du, ud))
    product(dwg, m, "dwg", (dg.t(), xd))
    product(dwu, m, "dwu", (du.t(), xd))

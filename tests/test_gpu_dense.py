"""Fully connected layers and gated blocks (dlf_linear, dlf_gated) and their backward passes against the formulas in 64 bits: both
types, sizes from one to beyond a tile, odd ones, strides, empty batches; sums that are exact, infinities, streams, graphs."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2011_05630_b200 import dense
from tests import dense_util as D

TYPES = [torch.float16, torch.bfloat16]
ids = lambda v: str(v).replace("torch.", "") if isinstance(v, torch.dtype) else None


class Maker:
    def __init__(self, seed, dtype):
        self.gen, self.dtype = torch.Generator(device="cuda").manual_seed(seed), dtype

    def mat(self, rows, cols, scale=1.0, pad=0, shift=0):
        """pad: further values between two rows, NaN; shift: values between the allocation's start and the matrix's."""
        t = torch.full((rows * (cols + pad) + shift,), float("nan"), device="cuda", dtype=self.dtype)
        m = t[shift:].view(rows, cols + pad)[:, :cols]
        m.copy_(torch.randn((rows, cols), generator=self.gen, device="cuda") * scale)
        return m

    def vec(self, n):
        return torch.randn((n,), generator=self.gen, device="cuda")


def check_linear(mk, m, k, n, a, bias, res, save, pads=(0, 0, 0), shift=0):
    x, w = mk.mat(m, k, pad=pads[0], shift=shift), mk.mat(n, k, k ** -0.5, pad=pads[1], shift=shift)
    b, r = mk.vec(n) if bias else None, mk.mat(m, n, pad=pads[2], shift=shift) if res else None
    got = dense.linear(x, w, b, r, act=a, save=save)
    y, z = got if save else (got, None)
    zr, zs, yr, ys = D.linear_ref(x, w, b, r, a)
    D.check(y, yr, ys, "y %s" % ((m, k, n, a),))
    if save:
        D.check(z, zr, zs, "z %s" % ((m, k, n, a),))


def check_linear_backward(mk, m, k, n, a, bias, res, pads=(0, 0, 0), shift=0):
    dy, x, w = mk.mat(m, n, pad=pads[2], shift=shift), mk.mat(m, k, pad=pads[0], shift=shift), mk.mat(n, k, k ** -0.5, pad=pads[1], shift=shift)
    z = mk.mat(m, n, 2.0, pad=pads[2], shift=shift) if a != "none" else None
    dx, dw, db, dr = dense.linear_backward(dy, x, w, z, act=a, bias=bias, residual=res)
    (d, s), = D.grad_ref(dy, z, None, a)
    off = D.through(d, s, dy.dtype, a != "none")
    xd, wd = x.double(), w.double()
    D.check(dx, d @ wd, off @ wd.abs() + D.sum_slack(n, d.abs() @ wd.abs()), "dx")
    D.check(dw, d.t() @ xd, off.t() @ xd.abs() + D.sum_slack(m, d.abs().t() @ xd.abs()), "dw")
    if bias:
        D.check(db, d.sum(0), s.sum(0) + D.sum_slack(m, d.abs().sum(0)), "db")
    if res and a == "none":
        assert dr is dy
    elif res:
        D.check(dr, d, s, "dr")


def check_gated(mk, m, k, n, a, bias, save, pads=(0, 0, 0), shift=0):
    x, wg, wu = mk.mat(m, k, pad=pads[0], shift=shift), mk.mat(n, k, k ** -0.5, pad=pads[1], shift=shift), mk.mat(n, k, k ** -0.5, pad=pads[2], shift=shift)
    bg, bu = (mk.vec(n), mk.vec(n)) if bias else (None, None)
    got = dense.gated(x, wg, wu, bg, bu, act=a, save=save)
    h, g, u = got if save else (got, None, None)
    gr, gs, ar, as_ = D.linear_ref(x, wg, bg, None, a)
    ur, us, _, _ = D.linear_ref(x, wu, bu, None, "none")
    D.check(h, ar * ur, ar.abs() * us + as_ * ur.abs() + as_ * us + 2.0 ** -23 * (ar * ur).abs(), "h %s" % ((m, k, n, a),))
    if save:
        D.check(g, gr, gs, "g")
        D.check(u, ur, us, "u")


def check_gated_backward(mk, m, k, n, a, bias, pads=(0, 0, 0), shift=0):
    dh, x = mk.mat(m, n, pad=pads[2], shift=shift), mk.mat(m, k, pad=pads[0], shift=shift)
    wg, wu = mk.mat(n, k, k ** -0.5, pad=pads[1], shift=shift), mk.mat(n, k, k ** -0.5, shift=shift)
    g, u = mk.mat(m, n, pad=pads[1], shift=shift), mk.mat(m, n, shift=shift)
    dx, dwg, dwu, dbg, dbu = dense.gated_backward(dh, x, wg, wu, g, u, act=a, bias=bias)
    (dg, sg), (du, su) = D.grad_ref(dh, g, u, a)
    og, ou = D.through(dg, sg, dh.dtype, True), D.through(du, su, dh.dtype, True)
    xd, gd, ud = x.double(), wg.double(), wu.double()
    D.check(dx, dg @ gd + du @ ud, og @ gd.abs() + ou @ ud.abs() + D.sum_slack(2 * n, dg.abs() @ gd.abs() + du.abs() @ ud.abs()), "dx")
    D.check(dwg, dg.t() @ xd, og.t() @ xd.abs() + D.sum_slack(m, dg.abs().t() @ xd.abs()), "dwg")
    D.check(dwu, du.t() @ xd, ou.t() @ xd.abs() + D.sum_slack(m, du.abs().t() @ xd.abs()), "dwu")
    if bias:
        D.check(dbg, dg.sum(0), sg.sum(0) + D.sum_slack(m, dg.abs().sum(0)), "dbg")
        D.check(dbu, du.sum(0), su.sum(0) + D.sum_slack(m, du.abs().sum(0)), "dbu")


SIZES = [(1, 1, 1), (40, 1, 1), (300, 1, 64), (300, 64, 1), (1, 8, 8), (1, 2048, 1000), (2, 64, 64), (3, 65, 63), (4, 1024, 256), (5, 100, 37), (7, 200, 130), (8, 512, 264), (9, 72, 1000), (15, 129, 257),
         (16, 4096, 512), (17, 640, 384), (32, 1160, 520), (33, 64, 2048), (63, 256, 256), (64, 2050, 128), (65, 96, 72), (100, 712, 129), (127, 128, 127),
         (128, 1088, 256), (129, 127, 255), (200, 333, 1000), (255, 64, 513), (256, 768, 768), (257, 520, 1032), (300, 1000, 1001), (520, 264, 136), (777, 1000, 300), (1030, 192, 2056)]


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear(size, dtype):
    mk = Maker(sum(size), dtype)
    check_linear(mk, *size, "none", False, False, False)
    check_linear(mk, *size, "gelu", True, True, True)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gated(size, dtype):
    mk = Maker(sum(size) + 1, dtype)
    check_gated(mk, *size, "silu", False, False)
    check_gated(mk, *size, "gelu_tanh", True, True)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear_backward(size, dtype):
    mk = Maker(sum(size) + 2, dtype)
    check_linear_backward(mk, *size, "none", True, True)
    check_linear_backward(mk, *size, "gelu", True, True)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gated_backward(size, dtype):
    mk = Maker(sum(size) + 3, dtype)
    check_gated_backward(mk, *size, "silu", False)
    check_gated_backward(mk, *size, "gelu_tanh", True)


@pytest.mark.parametrize("a", ["none", "relu", "relu6", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("m", [3, 40, 300])
def test_activations(m, a):
    mk = Maker(m, torch.bfloat16)
    check_linear(mk, m, 136, 200, a, True, True, True)
    check_linear_backward(mk, m, 136, 200, a, True, True)
    check_gated(mk, m, 136, 200, a, True, True)
    check_gated_backward(mk, m, 136, 200, a, True)


@pytest.mark.parametrize("pads,shift", [((8, 8, 8), 0), ((24, 0, 16), 8), ((1, 3, 5), 0), ((0, 0, 0), 1), ((8, 7, 8), 4)], ids=str)
@pytest.mark.parametrize("size", [(1, 256, 128), (6, 250, 136), (48, 264, 130), (260, 200, 264)], ids=str)
def test_strides(size, pads, shift):
    """Rows of a wider tensor (with NaN between them), rows and starts off the 16-byte boundaries."""
    mk = Maker(sum(size) + shift, torch.float16)
    check_linear(mk, *size, "silu", True, True, True, pads, shift)
    check_linear_backward(mk, *size, "silu", True, True, pads, shift)
    check_linear_backward(mk, *size, "none", True, True, pads, shift)
    check_gated(mk, *size, "silu", True, True, pads, shift)
    check_gated_backward(mk, *size, "silu", True, pads, shift)


@pytest.mark.parametrize("size", [(1, 250, 130), (10, 250, 130), (48, 122, 258), (300, 506, 1002)], ids=str)
def test_rows_that_end_inside_16_bytes(size):
    """Rows that start on 16-byte boundaries and end between two, NaN behind them."""
    mk, pads = Maker(sum(size), torch.bfloat16), (6, 6, 6)
    check_linear(mk, *size, "gelu", True, True, True, pads)
    check_linear_backward(mk, *size, "gelu", True, True, pads)
    check_linear_backward(mk, *size, "none", True, True, pads)
    check_gated(mk, *size, "silu", True, True, pads)
    check_gated_backward(mk, *size, "silu", True, pads)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("size", [(1, 512, 300), (8, 1000, 264), (24, 1100, 530), (130, 640, 300), (515, 600, 1000)], ids=str)
def test_exact_sums(size, dtype):
    """Small whole numbers: every sum is exact in fp32 in any order, so that the result is the exact one, rounded."""
    m, k, n = size
    gen = torch.Generator(device="cuda").manual_seed(k)
    whole = lambda *s: torch.randint(-2, 3, s, generator=gen, device="cuda").to(dtype)
    x, w, wu, r, dy = whole(m, k), whole(n, k), whole(n, k), whole(m, n), whole(m, n)
    b = torch.randint(-4, 5, (n,), generator=gen, device="cuda").float()
    want = x.double() @ w.double().t() + b.double() + r.double()
    assert torch.equal(dense.linear(x, w, b, r), want.to(dtype))
    dx, dw, db, dr = dense.linear_backward(dy, x, w)
    assert torch.equal(dx, (dy.double() @ w.double()).to(dtype)) and torch.equal(dw, (dy.double().t() @ x.double()).to(dtype))
    assert torch.equal(db.double(), dy.double().sum(0))
    h, g, u = dense.gated(x, w, wu, act="none", save=True)
    gd, ud = x.double() @ w.double().t(), x.double() @ wu.double().t()
    assert torch.equal(g, gd.to(dtype)) and torch.equal(u, ud.to(dtype)) and torch.equal(h, (gd * ud).to(dtype))


def test_rows_behind_the_last_are_left_alone():
    mk = Maker(5, torch.float16)
    for m, n in ((1, 130), (9, 136), (70, 256), (130, 264)):
        x, w = mk.mat(m, 256), mk.mat(n, 256, 1 / 16)
        buf = torch.full((m + 3, n + 8), 7.0, device="cuda", dtype=torch.float16)
        dense.linear(x, w, out=buf[:m, :n])
        assert bool((buf[m:] == 7).all()) and bool((buf[:, n:] == 7).all())
        assert torch.equal(buf[:m, :n], dense.linear(x, w))
        buf.fill_(7.0)
        dense.gated(x, w, w, out=buf[:m, :n])
        assert bool((buf[m:] == 7).all()) and bool((buf[:, n:] == 7).all())


@pytest.mark.parametrize("m", [2, 50, 300])
def test_output_over_the_residual(m):
    mk = Maker(m, torch.bfloat16)
    x, w, r = mk.mat(m, 320), mk.mat(264, 320, 0.05), mk.mat(m, 264)
    want = dense.linear(x, w, residual=r)
    assert dense.linear(x, w, residual=r, out=r) is r and torch.equal(r, want)


def test_no_rows():
    mk = Maker(1, torch.float16)
    w, x, dy = mk.mat(40, 64), torch.empty((0, 64), device="cuda", dtype=torch.float16), torch.empty((0, 40), device="cuda", dtype=torch.float16)
    assert dense.linear(x, w, mk.vec(40), save=True)[1].shape == (0, 40) and dense.gated(x, w, w).shape == (0, 40)
    dx, dw, db, dr = dense.linear_backward(dy, x, w, dy, act="gelu")
    assert dx.shape == (0, 64) and not bool(dw.any()) and not bool(db.any())
    dx, dwg, dwu, dbg, dbu = dense.gated_backward(dy, x, w, w, dy, dy, bias=True)
    assert dx.shape == (0, 64) and not bool(dwg.any()) and not bool(dwu.any()) and not bool(dbg.any()) and not bool(dbu.any())


@pytest.mark.parametrize("m", [1, 20, 200])
def test_infinities_and_nan_stay_in_their_rows(m):
    mk = Maker(m, torch.bfloat16)
    x, w = mk.mat(m, 200, pad=8), mk.mat(300, 200, 0.07)
    clean = dense.linear(x, w), dense.gated(x, w, w)
    row = m // 2
    x[row, 3], x[row, 7] = float("inf"), float("nan")
    for before, after in zip(clean, (dense.linear(x, w), dense.gated(x, w, w))):
        assert bool(torch.isnan(after[row]).all())
        keep = [i for i in range(m) if i != row]
        assert torch.equal(before[keep], after[keep])
    assert bool((dense.linear(x, w, act="relu")[row] == 0).all()) and bool((dense.linear(x, w, act="relu6")[row] == 0).all())   # (as in every kernel here)


@pytest.mark.parametrize("a", ["relu6", "gelu", "gelu_tanh", "silu"])
def test_large_and_small_values(a):
    """Sums of any size a bf16 can hold: activations and their derivatives at both ends, and at nothing."""
    v = torch.tensor([0.0, -0.0, 1e-38, 1e-6, 0.5, 3.0, 5.99, 6.0, 8.0, 16.0, 40.0, 90.0, 1e4, 1e20, 1e38], device="cuda")
    v = torch.cat([v, -v]).to(torch.bfloat16)
    for m in (1, 30, 300):
        w = torch.zeros((v.numel(), 8), device="cuda", dtype=torch.bfloat16)
        w[:, 0] = v
        x = torch.zeros((m, 8), device="cuda", dtype=torch.bfloat16)
        x[:, 0] = 1.0
        y, z = dense.linear(x, w, act=a, save=True)
        assert torch.equal(z, v.expand(m, -1))
        want = D.act(v.double(), a).expand(m, -1)
        D.check(y, want, D.ACT_ERR * (want.abs() + v.double().abs().clamp(max=16.0)), "y")   # (from 16 on it is v or 0 to the last bit)
        dy = torch.ones_like(y)
        dr = dense.linear_backward(dy, None, None, z, act=a, bias=False, residual=True, need_dx=False, need_dw=False)[3]
        slope = D.act_grad(v.double().clamp(-1e6, 1e6), a).expand(m, -1)
        D.check(dr, slope, D.ACT_ERR * (1 + v.double().abs().clamp(max=16.0)).expand(m, -1), "slope")


@pytest.mark.parametrize("m", [200, 3001])
def test_dz_over_dy_and_over_z(m):
    """The C ABI lets dz take the place of dy or of z (3001 rows: more of a thread's than are on their way at a time)."""
    from paper_2011_05630_b200 import binding as B
    mk = Maker(3, torch.float16)
    k, n = 136, 264
    dy, x, w, z = mk.mat(m, n), mk.mat(m, k), mk.mat(n, k), mk.mat(m, n)
    want = dense.linear_backward(dy, x, w, z, act="gelu", residual=True)
    for place in (dy.clone(), z.clone()):
        d, zz = (place, z) if torch.equal(place, dy) else (dy, place)
        dx, dw = torch.empty_like(x), torch.empty_like(w)
        args = dense._LINEAR_GRAD.pack(0, B.DENSE_ACTS["gelu"], m, k, n, d.data_ptr(), x.data_ptr(), w.data_ptr(), zz.data_ptr(), dx.data_ptr(), dw.data_ptr(),
                                       0, place.data_ptr(), n, k, k, n, k, k, n)
        B._check(B.lib().dlf_linear_grad(args, None, 0, torch.cuda.current_stream().cuda_stream), "dlf_linear_grad")
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and torch.equal(place, want[3])
    dense.synchronize()


def test_captured_before_any_other_call():
    """A process whose first calls are captured ones."""
    code = """
import torch
from paper_2011_05630_b200 import dense
x, w = torch.ones((40, 512), device="cuda").half(), torch.ones((264, 512), device="cuda").half()
big = torch.ones((2048, 512), device="cuda").half()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    a, b, c = dense.linear(x, w), dense.gated(x[:3], w, w, act="relu"), dense.linear_backward(dense.linear(big, w), big, w)
g.replay()
dense.synchronize()
assert bool((a == 512).all()) and bool((c[0] == 264 * 512).all() | torch.isinf(c[0]).all()) and bool(torch.isinf(b).all())
print("captured")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("m", [4, 60, 400])
def test_parts_of_a_backward_pass(m):
    mk = Maker(m, torch.float16)
    dy, x, w, z = mk.mat(m, 136), mk.mat(m, 200), mk.mat(136, 200), mk.mat(m, 136)
    whole = dense.linear_backward(dy, x, w, z, act="silu", residual=True)
    assert torch.equal(dense.linear_backward(dy, None, w, z, act="silu", bias=False, need_dw=False)[0], whole[0])
    assert torch.equal(dense.linear_backward(dy, x, None, z, act="silu", bias=False, need_dx=False)[1], whole[1])
    only = dense.linear_backward(dy, x, w, z, act="silu", residual=True, need_dx=False, need_dw=False)
    assert only[0] is None and only[1] is None and torch.equal(only[2], whole[2]) and torch.equal(only[3], whole[3])
    wu, u = mk.mat(136, 200), mk.mat(m, 136)
    whole = dense.gated_backward(dy, x, w, wu, z, u, bias=True)
    assert torch.equal(dense.gated_backward(dy, None, w, wu, z, u, need_dw=False)[0], whole[0])
    part = dense.gated_backward(dy, x, None, None, z, u, bias=True, need_dx=False)
    assert part[0] is None and all(torch.equal(p, q) for p, q in zip(part[1:], whole[1:]))


def test_same_call_same_bits():
    for m in (1, 30, 500):
        mk = Maker(m, torch.bfloat16)
        dy, x, w, z = mk.mat(m, 1000), mk.mat(m, 712), mk.mat(1000, 712), mk.mat(m, 1000)
        first = [dense.linear(x, w), *dense.linear_backward(dy, x, w, z, act="gelu", residual=True), dense.gated(x, w, w)]
        for _ in range(3):
            again = [dense.linear(x, w), *dense.linear_backward(dy, x, w, z, act="gelu", residual=True), dense.gated(x, w, w)]
            assert all(torch.equal(p, q) for p, q in zip(first, again))


def block(x, r, wg, wu, wd, dy):
    """A feed-forward block and its backward pass, as a training step runs it: gated projections, the way back with the residual."""
    h, g, u = dense.gated(x, wg, wu, save=True)
    y = dense.linear(h, wd, residual=r)
    dh, dwd, _, dr = dense.linear_backward(dy, h, wd, bias=False, residual=True)
    dx, dwg, dwu, _, _ = dense.gated_backward(dh, x, wg, wu, g, u)
    return y, dx, dwg, dwu, dwd


@pytest.mark.parametrize("m", [1, 24, 300])
def test_a_block_trains(m):
    """A block forwards and backwards against its formulas in 64 bits, and those against the difference quotient of the block."""
    mk = Maker(m, torch.float16)
    k, n = 256, 704
    x, wg, wu, wd = mk.mat(m, k), mk.mat(n, k, k ** -0.5), mk.mat(n, k, k ** -0.5), mk.mat(k, n, n ** -0.5)
    dy = mk.mat(m, k, 0.5)
    got = block(x, x, wg, wu, wd, dy)
    leaves = [t.double() for t in (x, wg, wu, wd)]
    f = lambda p: (D.act(p[0] @ p[1].t(), "silu") * (p[0] @ p[2].t())) @ p[3].t()
    xd, gd, ud, dd, e = *leaves, dy.double()
    g, u = xd @ gd.t(), xd @ ud.t()
    a, da = D.act(g, "silu"), D.act_grad(g, "silu")
    h, dh = a * u, e @ dd
    dg, du = dh * u * da, dh * a
    want = [h @ dd.t() + xd, dg @ gd + du @ ud, dg.t() @ xd, du.t() @ xd, e.t() @ h]
    for i, t in enumerate(want[1:]):
        d = torch.randn(t.shape, generator=mk.gen, device="cuda").double()
        step = 1e-5
        lo, hi = ([l + s * step * d if j == i else l for j, l in enumerate(leaves)] for s in (-1, 1))
        quotient = float(((f(hi) - f(lo)) * e).sum() / (2 * step))
        assert abs(float((t * d).sum()) - quotient) <= 1e-6 * float((t * d).abs().sum()), i   # (third derivatives of order 1 times 1e-10, 1e-16 / 1e-5)
    # roundings to 16 bits on the way, each half a step of its value, carried on by the formulas' derivatives (SILU's second one is below
    # 0.51), and the sums in fp32; 1.02: products of two of these
    r = D.half(torch.float16)
    sums = lambda k, p, q: D.sum_slack(k, p.abs() @ q.abs())
    odh = r * dh.abs() + sums(k, e, dd)
    og, ou = r * g.abs() + sums(k, xd, gd.t()), r * u.abs() + sums(k, xd, ud.t())
    oh = r * h.abs() + og * 1.1 * u.abs() + ou * a.abs()
    odg = odh * (u * da).abs() + (dh * da).abs() * ou + (dh * u).abs() * 0.51 * og + r * dg.abs()
    odu = odh * a.abs() + dh.abs() * 1.1 * og + r * du.abs()
    slack = [oh @ dd.abs().t() + sums(n, h, dd.t()), odg @ gd.abs() + odu @ ud.abs() + sums(2 * n, dg, gd) + sums(2 * n, du, ud),
             odg.t() @ xd.abs() + sums(m, dg.t(), xd), odu.t() @ xd.abs() + sums(m, du.t(), xd), e.abs().t() @ oh + sums(m, e.t(), h)]
    for name, t, w, s in zip(("y", "dx", "dwg", "dwu", "dwd"), got, want, slack):
        D.check(t, w, 1.02 * s + 1e-6, name)   # (1e-6: the activation's fp32 arithmetic, 2^-18 of values below 4, some of them at a time)


def test_streams_and_graphs():
    """Two captured blocks and eager ones on two streams, interleaved: each has its own results."""
    mk = Maker(9, torch.bfloat16)
    k, n = 512, 1408
    sets = [[mk.mat(m, k), mk.mat(m, k), mk.mat(n, k, k ** -0.5), mk.mat(n, k, k ** -0.5), mk.mat(k, n, n ** -0.5), mk.mat(m, k)] for m in (5, 300)]
    want = [block(*s) for s in sets]
    graphs, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(block(*s))
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(4):
        eager = []
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                graphs[i].replay()
                eager.append(block(*sets[1 - i]))
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(p, q) for p, q in zip(outs[i], want[i]))
            assert all(torch.equal(p, q) for p, q in zip(eager[i], want[1 - i]))
            for t in outs[i]:
                t.zero_()
        torch.cuda.synchronize()


def test_two_threads_at_once():
    """Two host threads, a stream each, the same calls over and over: each has its own results."""
    import threading
    k, n = 320, 712
    sets, want = [], []
    for m in (3, 90):
        mk = Maker(m, torch.float16)
        sets.append([mk.mat(m, k), mk.mat(m, k), mk.mat(n, k, k ** -0.5), mk.mat(n, k, k ** -0.5), mk.mat(k, n, n ** -0.5), mk.mat(m, k)])
        want.append(block(*sets[-1]))
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(30):
                    got = block(*sets[i])
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(p, q) for p, q in zip(got, want[i])):
                    wrong.append(i)
        except Exception as e:
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong


def test_wrong_tensors_are_refused():
    mk = Maker(1, torch.float16)
    x, w, y = mk.mat(4, 64), mk.mat(40, 64), mk.mat(4, 40)
    for f in (lambda: dense.linear(x, w.bfloat16()), lambda: dense.linear(x.float(), w), lambda: dense.linear(x, mk.mat(40, 56)), lambda: dense.linear(x[0], w),
              lambda: dense.linear(x, mk.mat(64, 40).t()), lambda: dense.linear(x[:1].expand(4, 64), w), lambda: dense.linear(x, w, act="tanh"),
              lambda: dense.linear(x, w, bias=y[0]), lambda: dense.linear(x, w, bias=mk.vec(80)[::2]), lambda: dense.linear(x, w, residual=mk.mat(4, 41)),
              lambda: dense.linear(x, w, out=mk.mat(5, 40)), lambda: dense.linear(x, w.cpu()), lambda: dense.linear_backward(y, x, w, act="gelu"),
              lambda: dense.linear_backward(y, None, w), lambda: dense.linear_backward(y, x, None), lambda: dense.gated(x, w, mk.mat(41, 64)),
              lambda: dense.gated_backward(y, x, w, w, y, None), lambda: dense.gated_backward(y, x, None, w, y, y)):
        with pytest.raises(ValueError):
            f()
    from paper_2011_05630_b200 import binding as B
    for f in (lambda: dense.linear(x, mk.mat(0, 64)), lambda: dense.linear(mk.mat(4, 0), mk.mat(40, 0)), lambda: dense.linear(x, mk.mat(64, 64), out=x)):
        with pytest.raises(B.DlfError):
            f()
    dense.synchronize()


def test_offsets_beyond_32_bits():
    """Two thousand million values in an output and in the residual; the last rows are where an offset of 32 bits goes wrong."""
    m, k, n = 270000, 64, 8192
    if torch.cuda.get_device_properties(0).total_memory < 60 << 30:
        pytest.skip("needs 30 GB")
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((m, k), generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    w = (torch.randn((n, k), generator=gen, device="cuda") / 8).to(torch.bfloat16)
    y = torch.zeros((m, n), device="cuda", dtype=torch.bfloat16)
    y[-2:] = 1.0
    dense.linear(x, w, residual=y, out=y)
    tail = slice(m - 300, m)
    r = torch.zeros((300, n), device="cuda", dtype=torch.bfloat16)
    r[-2:] = 1.0
    z, s, _, _ = D.linear_ref(x[tail], w, None, r, "none")
    D.check(y[tail], z, s, "y")
    dx, _, db, _ = dense.linear_backward(y, None, w, y, act="relu", need_dw=False)
    (d, ds), = D.grad_ref(y[tail], y[tail], None, "relu")
    D.check(dx[tail], d @ w.double(), D.through(d, ds, y.dtype, True) @ w.double().abs() + D.sum_slack(n, d.abs() @ w.double().abs()), "dx")
    assert bool(torch.isfinite(db).all())

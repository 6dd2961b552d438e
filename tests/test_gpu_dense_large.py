"""Dense operators on matrices of more than 2^31 values (2^32 bytes): weights and their gradients, inputs and theirs.  Gradients that are 0 but in the last
rows or columns leave sums that only what lies behind those offsets enters; small whole numbers make them exact."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2011_05630_b200 import dense

LONG, SHORT, TAIL = 1060000, 2048, 300
assert LONG * SHORT > 1 << 31


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.get_device_properties(0).total_memory < 100 << 30:
        pytest.skip("needs 60 GB")
    yield
    torch.cuda.empty_cache()


def whole(gen, rows, cols, pad=0, shift=0):
    """Small whole numbers in rows `pad` values apart, `shift` values from the start of their memory."""
    t = torch.randint(-2, 3, (shift + rows * (cols + pad),), generator=gen, device="cuda", dtype=torch.int8).to(torch.bfloat16)
    return t[shift:].view(rows, cols + pad)[:, :cols]


def only_tail(t, dim):
    t.narrow(dim, 0, t.shape[dim] - TAIL).zero_()
    return t


@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 1)], ids=["aligned", "anywhere"])
@pytest.mark.parametrize("m", [4, 40, 600])
def test_weights(m, pad, shift):
    gen = torch.Generator(device="cuda").manual_seed(m)
    x, w, wu = whole(gen, m, SHORT), whole(gen, LONG, SHORT, pad, shift), whole(gen, LONG, SHORT, pad, shift)
    xd, wd, ud = x.double(), w[-TAIL:].double(), wu[-TAIL:].double()
    g, u = xd @ wd.t(), xd @ ud.t()
    assert torch.equal(dense.linear(x, w)[:, -TAIL:], g.bfloat16())
    assert torch.equal(dense.gated(x, w, wu, act="relu")[:, -TAIL:], (g.relu() * u).bfloat16())
    dy, z = only_tail(whole(gen, m, LONG), 1), whole(gen, m, LONG)
    d, e, zd = dy[:, -TAIL:].double(), z[:, -TAIL:].double(), (z[:, -TAIL:] > 0).double()
    dx, dw, db, _ = dense.linear_backward(dy, x, w, z, act="relu")
    assert torch.equal(dx, ((d * zd) @ wd).bfloat16()) and torch.equal(dw[-TAIL:], ((d * zd).t() @ xd).bfloat16())
    assert torch.equal(db[-TAIL:].double(), (d * zd).sum(0)) and not bool(db[:-TAIL].any()) and not bool(dw[:-TAIL].any())
    del dw
    dx, dwg, dwu, _, _ = dense.gated_backward(dy, x, w, wu, z, z, act="relu")
    dg, du = d * e * zd, d * e.relu()
    assert torch.equal(dx, (dg @ wd + du @ ud).bfloat16())
    assert torch.equal(dwg[-TAIL:], (dg.t() @ xd).bfloat16()) and torch.equal(dwu[-TAIL:], (du.t() @ xd).bfloat16())


@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 1)], ids=["aligned", "anywhere"])
@pytest.mark.parametrize("n", [33, 64])
def test_rows(n, pad, shift):
    """A long batch: x and its gradient."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, w, wu = whole(gen, LONG, SHORT, pad, shift), whole(gen, n, SHORT), whole(gen, n, SHORT)
    xd, wd, ud = x[-TAIL:].double(), w.double(), wu.double()
    g, u = xd @ wd.t(), xd @ ud.t()
    assert torch.equal(dense.linear(x, w)[-TAIL:], g.bfloat16())
    assert torch.equal(dense.gated(x, w, wu, act="relu")[-TAIL:], (g.relu() * u).bfloat16())
    dy, z = only_tail(whole(gen, LONG, n), 0), whole(gen, LONG, n)
    d, e, zd = dy[-TAIL:].double(), z[-TAIL:].double(), (z[-TAIL:] > 0).double()
    dx, dw, db, _ = dense.linear_backward(dy, x, w, z, act="relu")
    assert torch.equal(dx[-TAIL:], ((d * zd) @ wd).bfloat16()) and not bool(dx[:-TAIL].any())
    assert torch.equal(dw, ((d * zd).t() @ xd).bfloat16()) and torch.equal(db.double(), (d * zd).sum(0))
    del dx
    dx, dwg, dwu, _, _ = dense.gated_backward(dy, x, w, wu, z, z, act="relu")
    dg, du = d * e * zd, d * e.relu()
    assert torch.equal(dx[-TAIL:], (dg @ wd + du @ ud).bfloat16())
    assert torch.equal(dwg, (dg.t() @ xd).bfloat16()) and torch.equal(dwu, (du.t() @ xd).bfloat16())

"""Activations of the dense operators where they are small: each is its formula's value to a share of the value itself, which a bound on
the error beside the sum would not show.

The exponentials' arguments are products of a few factors in fp32, each rounded: for GELU 2.5 roundings of an argument of at most 113
(v = -12.5), for SILU 1.5 of 115 (v = -80), for GELU_TANH 5.5 of 66 (v = -9); times ln 2 for the exponents of 2, these are shares of
1.2e-5, 7.2e-6 and 2.2e-5 of the result.  The functions themselves add 2^-20 at most: 2^-15 = 3.05e-5 in all."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2011_05630_b200 import dense
from tests import dense_util as D
from tests.test_gpu_dense import TYPES, ids

LEAST = {"gelu": -12.5, "silu": -80.0, "gelu_tanh": -9.0}
SHARE = 2.0 ** -15


def exact(v, a):
    """act(v) and act'(v) without a cancelled sum, and the sum of the absolute terms of act'(v)."""
    v = v.double()
    if a == "gelu":
        cdf, pdf = 0.5 * torch.special.erfc(-v / math.sqrt(2.0)), torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
        return v * cdf, cdf + v * pdf, cdf + (v * pdf).abs()
    t = v if a == "silu" else 2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)
    dt = 1.0 if a == "silu" else 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v * v)
    s, w = torch.sigmoid(t), torch.sigmoid(-t)
    return v * s, s + v * s * w * dt, s + (v * s * w * dt).abs()


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("m", [1, 30, 300])
@pytest.mark.parametrize("a", list(LEAST))
def test_small_values(a, m, dtype):
    v = torch.linspace(LEAST[a], 6.0, 2000, device="cuda").to(dtype)
    w = torch.zeros((v.numel(), 8), device="cuda", dtype=dtype)
    w[:, 0] = v
    x = torch.zeros((m, 8), device="cuda", dtype=dtype)
    x[:, 0] = 1.0
    one = torch.full((v.numel(), 8), 0.125, device="cuda", dtype=dtype)
    y, z = dense.linear(x, w, act=a, save=True)
    assert torch.equal(z, v.expand(m, -1))
    want, slope, terms = exact(v, a)
    D.check(y, want.expand(m, -1), SHARE * want.abs().expand(m, -1), "y")
    h = dense.gated(x, w, one, act=a)   # (u = 1/8)
    D.check(h, 0.125 * want.expand(m, -1), 0.125 * SHARE * want.abs().expand(m, -1), "h")
    dr = dense.linear_backward(torch.ones_like(y), None, None, z, act=a, bias=False, residual=True, need_dx=False, need_dw=False)[3]
    D.check(dr, slope.expand(m, -1), SHARE * terms.expand(m, -1), "slope")

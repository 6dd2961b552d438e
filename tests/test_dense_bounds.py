"""The bound on the root mean square tells a second rounding from the documented ones (planted here, in 64-bit arithmetic on the CPU)."""
import pytest

torch = pytest.importorskip("torch")

from tests import dense_bounds as R, dense_util as D


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["float16", "bfloat16"])
@pytest.mark.parametrize("k", [64, 128, 200])
def test_a_second_rounding_shows(k, dtype):
    gen = torch.Generator().manual_seed(k)
    mat = lambda r, c: torch.randn((r, c), generator=gen, dtype=torch.float64)
    dy, z, w = mat(96, k).to(dtype), mat(96, k).to(dtype), mat(k, 160).to(dtype).double()
    d = dy.double() * D.act_grad(z.double(), "gelu")
    once = R.rounded(d, dtype)
    want = once @ w
    absum = once.abs() @ w.abs()
    R.check_rms(want.to(dtype), want, k, absum, "as documented")
    with pytest.raises(AssertionError):   # the slope rounded before the gradient is
        R.check_rms((R.rounded(dy.double() * R.rounded(D.act_grad(z.double(), "gelu"), dtype), dtype) @ w).to(dtype), want, k, absum, "")
    with pytest.raises(AssertionError):   # the result rounded, and a residual of no size added to that
        R.check_rms(R.rounded(want + 0.37 * want, dtype).sub(R.rounded(0.37 * want, dtype)).to(dtype), want, k, absum, "")
    u = mat(96, k) @ w
    h = D.act(want, "silu") * u
    R.check_rms(h.to(dtype), h, 0, torch.zeros(1), "a product of two sums")
    with pytest.raises(AssertionError):   # one of the sums rounded before the product
        R.check_rms((D.act(want, "silu") * R.rounded(u, dtype)).to(dtype), h, 0, torch.zeros(1), "")

"""The dense operators' formulas in 64 bits, and how far a result may be from them by arithmetic.

A product's sum of K terms in fp32 is off by at most K steps of 2^-23 of the sum of the terms' absolute values (additions that may
truncate); a value rounded to 16 bits by half a step, eps / 2 of it.  Activations are 1.13-Lipschitz (GELU's largest slope is 1.129),
their derivatives 1.6-Lipschitz; both are computed in fp32 from functions that are good to 2^-20 (exp at the arguments that
matter, the quotient, erf)."""
import math

import torch

ACT_ERR = 2.0 ** -18   # a few operations on functions good to 2^-20
LIP = 1.13


def act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "relu6":
        return torch.where(z > 0, z, torch.zeros_like(z)).clamp(max=6.0)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def act_grad(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "relu6":
        return ((z > 0) & (z < 6)).to(z.dtype)
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c, a = math.sqrt(2.0 / math.pi), 0.044715
        t = torch.tanh(c * (z + a * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * a * z * z)
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    return torch.ones_like(z)


def half(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps   # a subnormal step


def check(got, want, slack, what):
    """Every element: rounded once (half a step), and `slack` before that."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    g = got.double()
    bound = half(got.dtype) * (want.abs() + slack) + slack + tiny(got.dtype)
    off = (g - want).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        i = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError("%s: %d of %d off; first at %s: got %g want %g bound %g" % (what, int(bad.sum()), bad.numel(), i, g[i], want[i], bound[i]))


def sum_slack(k, absum):
    return k * 2.0 ** -23 * absum


def linear_ref(x, w, b, r, a):
    """(z, its slack, y, its slack)"""
    xd, wd = x.double(), w.double()
    z, s = xd @ wd.t(), sum_slack(x.shape[1] + 2, xd.abs() @ wd.abs().t())
    if b is not None:
        z, s = z + b.double(), s + 2.0 ** -23 * b.double().abs()
    if r is not None:
        z, s = z + r.double(), s + 2.0 ** -23 * r.double().abs()
    y = act(z, a)
    return z, s, y, LIP * s + ACT_ERR * (y.abs() + z.abs()) * (a not in ("none", "relu", "relu6"))


def grad_ref(dy, z, u, a):
    """[(d, slack in fp32)] behind the activation: one of a linear layer (u None), two of a gated block."""
    dyd = dy.double()
    zd = z.double() if z is not None else torch.zeros_like(dyd)
    err = ACT_ERR * (a not in ("none", "relu", "relu6"))
    if u is None:
        d = dyd * act_grad(zd, a)
        return [(d, dyd.abs() * err * (1 + zd.abs()) + d.abs() * 2.0 ** -23)]
    ud = u.double()
    d, e = dyd * ud * act_grad(zd, a), dyd * act(zd, a)
    return [(d, (dyd * ud).abs() * err * (1 + zd.abs()) + d.abs() * 2.0 ** -22), (e, dyd.abs() * err * (zd.abs() + e.abs()) + e.abs() * 2.0 ** -22)]


def through(d, slack, dtype, rounded):
    """How far a gradient's elements may be off as a product's operand: rounded to 16 bits, or as they came."""
    return slack + (half(dtype) * (d.abs() + slack) + tiny(dtype) if rounded else 0.0)

"""The work of the dense operators whose speed counts: a fully connected layer with bias, residual and activation in its
epilogue, a gated feed-forward block's two projections with activation and product, and the backward pass of both, from one
token to long sequences.

    linear            y = act(x W^T + b + r), optionally with the sum z = x W^T + b + r that a backward pass needs
    linear_backward   dz = dy act'(z);  dx = dz W,  dW = dz^T x,  db = sum over rows of dz,  dr = dz
    gated             g = x Wg^T + bg,  u = x Wu^T + bu,  h = act(g) u, optionally with g and u
    gated_backward    dg = dh u act'(g),  du = dh act(g);  dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x,  dbg, dbu

Matrices are fp16 or bf16, weights [out][in], biases and their gradients fp32, sums in fp32; z, g and u are what the forward pass
kept, in the matrices' type.  Activations are N(0, 1), weights N(0, 1/fan_in), biases N(0, 0.01), all drawn on the GPU from the
seed.  `pad` is how much longer than its columns a row of x lies in memory (x is part of a wider tensor).
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
_ACTS = ("none", "relu", "relu6", "gelu", "gelu_tanh", "silu")
_MAX_FLOPS = 2.0e12     # of a drawn case: no more than the largest listed one has
_MAX_BYTES = 5.0e8


def listed():
    def linear(name, m, k, n, dtype, act="none", bias=True, residual=False, save=False, pad=0):
        return {"name": name, "kind": "linear", "m": m, "k": k, "n": n, "dtype": dtype, "act": act, "bias": bias,
                "residual": residual, "save": save, "pad": pad}

    def linear_bwd(name, m, k, n, dtype, act="none", bias=True, residual=False, pad=0):
        return {"name": name, "kind": "linear_backward", "m": m, "k": k, "n": n, "dtype": dtype, "act": act, "bias": bias,
                "residual": residual, "pad": pad}

    def gated(name, m, k, f, dtype, act="silu", bias=False, save=False, pad=0):
        return {"name": name, "kind": "gated", "m": m, "k": k, "n": f, "dtype": dtype, "act": act, "bias": bias, "save": save, "pad": pad}

    def gated_bwd(name, m, k, f, dtype, act="silu", bias=False, pad=0):
        return {"name": name, "kind": "gated_backward", "m": m, "k": k, "n": f, "dtype": dtype, "act": act, "bias": bias, "pad": pad}

    return [
        # the classifier head of the repository's residual networks on one image: the smallest call, launch latency is all there is
        linear("linear_1x2048x1000", 1, 2048, 1000, "fp16"),
        # a feed-forward block's way back to the model width for four sequences that get a token each: weights are streamed
        linear("linear_4x11264x4096_res", 4, 11264, 4096, "bf16", bias=False, residual=True),
        # the repository's first fully connected layer behind a convolution, at its batch of 32: weights again, tensor cores needed
        linear("linear_32x9216x4096_relu", 32, 9216, 4096, "fp16", act="relu"),
        # a batch of ragged length through a layer whose sizes divide by nothing, kept for a backward pass; x is part of a wider tensor
        linear("linear_777x1000x1001_gelu", 777, 1000, 1001, "bf16", act="gelu", residual=True, save=True, pad=24),
        # prefill of long prompts, the way back to the model width with the residual stream: bound by the tensor cores
        linear("linear_8192x11264x4096_res", 8192, 11264, 4096, "bf16", bias=False, residual=True),
        # training step of a plain feed-forward layer, its activation's derivative included
        linear_bwd("linear_bwd_4096x2048x8192_gelu", 4096, 2048, 8192, "bf16", act="gelu"),
        # training step of a classifier head on a small batch
        linear_bwd("linear_bwd_200x2048x1000", 200, 2048, 1000, "fp16"),
        # a token of one sequence: two weight matrices are read, and little else
        gated("gated_1x4096x11264", 1, 4096, 11264, "bf16"),
        # a token each for the sequences of a batch
        gated("gated_24x2048x5632", 24, 2048, 5632, "fp16"),
        # prefill of long prompts: bound by the tensor cores, the largest call
        gated("gated_8192x4096x14336", 8192, 4096, 14336, "bf16"),
        # a ragged batch of training tokens, the forward pass's two sums in hand, sizes that divide by nothing
        gated_bwd("gated_bwd_333x1000x2731_bias", 333, 1000, 2731, "fp16", act="gelu_tanh", bias=True),
        # training step of a gated block of ordinary size
        gated_bwd("gated_bwd_4096x2048x5632", 4096, 2048, 5632, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A layer's width: mostly whole multiples of 64, sometimes of 8, sometimes as odd as it comes."""
    v, how = _log_int(rng, lo, hi), rng.random()
    if how < 0.5:
        return max(64, v // 64 * 64)
    return max(8, v // 8 * 8) if how < 0.75 else v


def draw(rng):
    while True:
        kind = rng.choice(["linear", "linear", "linear_backward", "gated", "gated", "gated_backward"])
        case = {"kind": kind, "m": _log_int(rng, 1, 8192), "k": _width(rng, 64, 16384), "n": _width(rng, 64, 16384),
                "dtype": rng.choice(["fp16", "bf16", "bf16"]), "act": rng.choice(_ACTS if kind.startswith("linear") else ("silu", "silu", "gelu", "gelu_tanh", "relu")),
                "bias": rng.random() < 0.5, "pad": rng.choice([0, 0, 0, 8, 40])}
        if kind.startswith("linear"):
            case["residual"] = rng.random() < 0.5
        if not kind.endswith("backward"):
            case["save"] = rng.random() < 0.3
        w = work(case)
        if w["flops"] <= _MAX_FLOPS and w["bytes"] <= _MAX_BYTES:
            return case


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, m, k, n = _TYPES[case["dtype"]], case["m"], case["k"], case["n"]

    def normal(rows, cols, scale=1.0, pad=0):
        t = torch.randn((rows, cols + pad), generator=gen, device="cuda").mul_(scale).to(dtype)
        return t[:, :cols]

    def bias():
        return torch.randn((n,), generator=gen, device="cuda").mul_(0.1) if case["bias"] else None

    state = {"case": case, "x": normal(m, k, pad=case["pad"])}
    x = state["x"]
    if case["kind"].startswith("linear"):
        state["w"], state["b"] = normal(n, k, k ** -0.5), bias()
        state["r"] = normal(m, n) if case["residual"] else None
        if case["kind"] == "linear_backward":
            state["dy"] = normal(m, n)
            if case["act"] != "none":   # what the forward pass kept
                z = (x @ state["w"].t()).float()
                z = z if state["b"] is None else z + state["b"]
                state["z"] = (z if state["r"] is None else z + state["r"].float()).to(dtype)
            state["r"] = None
    else:
        state["wg"], state["wu"], state["bg"], state["bu"] = normal(n, k, k ** -0.5), normal(n, k, k ** -0.5), bias(), bias()
        if case["kind"] == "gated_backward":
            state["dh"] = normal(m, n)
            for name, w, b in (("g", "wg", "bg"), ("u", "wu", "bu")):
                s = x @ state[w].t()
                state[name] = s if state[b] is None else (s.float() + state[b]).to(dtype)
    return state


def run(state):
    case = state["case"]
    return _own(case, state) if own else _plain(case, state)


def _own(case, s):
    from paper_2011_05630_b200 import dense
    if case["kind"] == "linear":
        return dense.linear(s["x"], s["w"], s["b"], s["r"], act=case["act"], save=case["save"])
    if case["kind"] == "linear_backward":
        return dense.linear_backward(s["dy"], s["x"], s["w"], s.get("z"), act=case["act"], bias=case["bias"], residual=case["residual"])
    if case["kind"] == "gated":
        return dense.gated(s["x"], s["wg"], s["wu"], s["bg"], s["bu"], act=case["act"], save=case["save"])
    return dense.gated_backward(s["dh"], s["x"], s["wg"], s["wu"], s["g"], s["u"], act=case["act"], bias=case["bias"])


# ---- the plain form: elementary operations in 32 bits, rounded once at the end ------------------------------------------------


def _act(z, act):
    """act(z) and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0.0), (z > 0).float()
    if act == "relu6":
        return z.clamp(0.0, 6.0), ((z > 0) & (z < 6)).float()
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return z * s, s * (1.0 + z * (1.0 - s))
    if act == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 0.134145 * z * z)


def _plain(case, s):
    dtype, act = _TYPES[case["dtype"]], case["act"]
    x = s["x"].float()
    if case["kind"] == "linear":
        z = x @ s["w"].float().t()
        if s["b"] is not None:
            z = z + s["b"]
        if s["r"] is not None:
            z = z + s["r"].float()
        y = _act(z, act)[0].to(dtype)
        return (y, z.to(dtype)) if case["save"] else y
    if case["kind"] == "linear_backward":
        dz = s["dy"].float()
        if act != "none":
            dz = dz * _act(s["z"].float(), act)[1]
        return ((dz @ s["w"].float()).to(dtype), (dz.t() @ x).to(dtype), dz.sum(0) if case["bias"] else None,
                dz.to(dtype) if case["residual"] else None)
    if case["kind"] == "gated":
        g, u = x @ s["wg"].float().t(), x @ s["wu"].float().t()
        if s["bg"] is not None:
            g, u = g + s["bg"], u + s["bu"]
        h = (_act(g, act)[0] * u).to(dtype)
        return (h, g.to(dtype), u.to(dtype)) if case["save"] else h
    a, da = _act(s["g"].float(), act)
    dh = s["dh"].float()
    dg, du = dh * s["u"].float() * da, dh * a
    return ((dg @ s["wg"].float() + du @ s["wu"].float()).to(dtype), (dg.t() @ x).to(dtype), (du.t() @ x).to(dtype),
            dg.sum(0) if case["bias"] else None, du.sum(0) if case["bias"] else None)


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------------


def _function(act):
    f = torch.nn.functional
    return {"none": lambda v: v * 1.0, "relu": f.relu, "relu6": f.relu6, "silu": f.silu, "gelu": f.gelu,
            "gelu_tanh": lambda v: f.gelu(v, approximate="tanh")}[act]


def exact(case, seed):
    s = {name: v.double() if isinstance(v, torch.Tensor) else v for name, v in prepare(case, seed).items()}
    fn = _function(case["act"])
    affine = lambda w, b: torch.nn.functional.linear(s["x"], s[w], s[b])
    if case["kind"] == "linear":
        z = affine("w", "b") + (0.0 if s["r"] is None else s["r"])
        return (fn(z), z) if case["save"] else fn(z)
    if case["kind"] == "gated":
        g, u = affine("wg", "bg"), affine("wu", "bu")
        return (fn(g) * u, g, u) if case["save"] else fn(g) * u
    if case["kind"] == "linear_backward":
        z = s["z"] if "z" in s else torch.zeros_like(s["dy"])
        leaf = z.requires_grad_(True)
        dz, = torch.autograd.grad(fn(leaf), leaf, s["dy"])
        return (torch.einsum("mn,nk->mk", dz, s["w"]), torch.einsum("mn,mk->nk", dz, s["x"]), dz.sum(0) if case["bias"] else None,
                dz if case["residual"] else None)
    g, u = s["g"].requires_grad_(True), s["u"].requires_grad_(True)
    dg, du = torch.autograd.grad(fn(g) * u, (g, u), s["dh"])
    both = torch.cat([dg, du], 1)
    return (both @ torch.cat([s["wg"], s["wu"]], 0), torch.einsum("mn,mk->nk", dg, s["x"]), torch.einsum("mn,mk->nk", du, s["x"]),
            dg.sum(0) if case["bias"] else None, du.sum(0) if case["bias"] else None)


def work(case):
    """Every input read once and every output written once; the products' multiplications and additions."""
    m, k, n = case["m"], case["k"], case["n"]
    bias = 4 * n if case["bias"] else 0
    if case["kind"] == "linear":
        return {"bytes": 2 * (m * k + n * k + m * n * (1 + case["residual"] + case["save"])) + bias, "flops": 2 * m * n * k}
    if case["kind"] == "linear_backward":
        maps = 1 + (case["act"] != "none") + (case["residual"] and case["act"] != "none")
        return {"bytes": 2 * (2 * m * k + 2 * n * k + m * n * maps) + bias, "flops": 4 * m * n * k}
    if case["kind"] == "gated":
        return {"bytes": 2 * (m * k + 2 * n * k + m * n * (1 + 2 * case["save"])) + 2 * bias, "flops": 4 * m * n * k}
    return {"bytes": 2 * (2 * m * k + 4 * n * k + 3 * m * n) + 2 * bias, "flops": 8 * m * n * k}

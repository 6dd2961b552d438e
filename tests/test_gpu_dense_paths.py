"""Every kernel and layout of the dense operators on the device, through the C interface: inputs with NaN between their rows, outputs with guards between
theirs, in front and behind, a workspace with a guard behind it.  Small whole numbers give sums that are exact in any order, so that a result is the
exact one, rounded; random numbers go through the smooth activations, within bounds by arithmetic."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2011_05630_b200 import binding as B, dense
from tests import dense_paths as P, dense_util as D

NAMES = {torch.float16: "f16", torch.bfloat16: "bf16"}
GUARD = 7.0


class Matrix:
    """rows x cols within `fill`: pad values between two rows, shift ahead of the first, 64 behind the last."""

    def __init__(self, rows, cols, pad, shift, fill, dtype):
        self.room = torch.full((shift + rows * (cols + pad) + 64,), fill, device="cuda", dtype=dtype)
        self.t = self.room[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]

    def only_written(self):
        """True if what is not the matrix is as it was."""
        self.t.fill_(GUARD)
        return bool((self.room == GUARD).all())


def run(case, dtype, values, act=None):
    """(inputs, outputs) of a call: values(rows, cols, name) makes an input."""
    outs = P.OUTPUTS[case.op].split()
    case = P.Case(case.name, case.op, case.m, case.k, case.n, case.expect, " ".join(case.without), case.pad, case.shift, case.out_pad, case.out_shift, act or case.act)
    mats = {t: Matrix(*size, GUARD if t in outs else float("nan"), dtype) for t, size in case.matrices().items()}
    vecs = {t: torch.full((case.n + 17,), GUARD, device="cuda") for t in case.vectors()}
    vec = lambda t: vecs[t][1:1 + case.n]   # (off the 16-byte boundaries)
    given = {}
    for t in mats:
        if t not in outs:
            mats[t].t.copy_(values(*mats[t].t.shape, t))
            given[t] = mats[t].t
    for t in vecs:
        if not t.startswith("d"):
            vec(t).copy_(values(1, case.n, t)[0])
            given[t] = vec(t)
    args = case.pack(NAMES[dtype], lambda t: vec(t).data_ptr() if t in vecs else mats[t].t.data_ptr())
    need = C.c_size_t()
    B._check(getattr(B.lib(), "dlf_%s_workspace_bytes" % case.op)(args, C.byref(need)), case.op)
    ws = torch.full((need.value + 512,), 255, device="cuda", dtype=torch.uint8)   # (NaN)
    B._check(getattr(B.lib(), "dlf_" + case.op)(args, ws.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream), case.op)
    dense.synchronize()
    got = {t: (mats[t].t if t in mats else vec(t)).clone() for t in mats.keys() | vecs.keys() if t in outs}
    assert bool((ws[need.value:] == 255).all()), (case.name, "behind the workspace")
    for t in got:
        if t in mats:
            assert mats[t].only_written(), (case.name, t, "beside the matrix")
        else:
            vec(t).fill_(GUARD)
            assert bool((vecs[t] == GUARD).all()), (case.name, t, "beside the vector")
    return given, got


def formulas(op, v, a):
    """The outputs in 64 bits, and how far fp32 sums and 16-bit operands may be off: name -> (value, slack)."""
    t = {name: x.double() for name, x in v.items()}
    if op == "linear":
        z, s, y, ys = D.linear_ref(v["x"], v["w"], v.get("bias"), v.get("res"), a)
        return {"z": (z, s), "y": (y, ys)}
    if op == "gated":
        g, gs, h, hs = D.linear_ref(v["x"], v["wg"], v.get("bg"), None, a)
        u, us, _, _ = D.linear_ref(v["x"], v["wu"], v.get("bu"), None, "none")
        return {"g": (g, gs), "u": (u, us), "h": (h * u, h.abs() * us + hs * u.abs() + hs * us + 2.0 ** -23 * (h * u).abs())}
    m, dtype = v["x"].shape[0], v["x"].dtype
    if op == "linear_grad":
        (d, s), = D.grad_ref(v["dy"], v["z"], None, a)
        off, n = D.through(d, s, dtype, True), d.shape[1]
        return {"dz": (d, s), "db": (d.sum(0), s.sum(0) + D.sum_slack(m, d.abs().sum(0))),
                "dx": (d @ t["w"], off @ t["w"].abs() + D.sum_slack(n, d.abs() @ t["w"].abs())),
                "dw": (d.t() @ t["x"], off.t() @ t["x"].abs() + D.sum_slack(m, d.abs().t() @ t["x"].abs()))}
    (dg, sg), (du, su) = D.grad_ref(v["dh"], v["g"], v["u"], a)
    og, ou, n = D.through(dg, sg, dtype, True), D.through(du, su, dtype, True), dg.shape[1]
    out = {"dx": (dg @ t["wg"] + du @ t["wu"], og @ t["wg"].abs() + ou @ t["wu"].abs() + D.sum_slack(2 * n, dg.abs() @ t["wg"].abs() + du.abs() @ t["wu"].abs()))}
    for name, d, s, o in (("g", dg, sg, og), ("u", du, su, ou)):
        out["dw" + name] = (d.t() @ t["x"], o.t() @ t["x"].abs() + D.sum_slack(m, d.abs().t() @ t["x"].abs()))
        out["db" + name] = (d.sum(0), s.sum(0) + D.sum_slack(m, d.abs().sum(0)))
    return out


GROUPS = {}
for c in P.CASES:
    GROUPS.setdefault("%s %s" % (c.op, c.expect.split(" out=")[0].replace("sources=1 ", "")), []).append(c)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["float16", "bfloat16"])
@pytest.mark.parametrize("group", list(GROUPS))
def test_exact_sums(group, dtype):
    for i, c in enumerate(GROUPS[group]):
        gen = torch.Generator(device="cuda").manual_seed(c.m + c.k + c.n)
        given, got = run(c, dtype, lambda r, q, name: torch.randint(-2, 3, (r, q), generator=gen, device="cuda").float())
        for name, (want, _) in formulas(c.op, given, c.act).items():
            assert float(want.abs().max()) < 2 ** 24
            assert torch.equal(got[name], want.to(got[name].dtype)), (c.name, name, c.expect)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["float16", "bfloat16"])
@pytest.mark.parametrize("group", list(GROUPS))
def test_random_numbers(group, dtype):
    for i, c in enumerate(GROUPS[group]):
        gen = torch.Generator(device="cuda").manual_seed(c.m + c.k + c.n + 1)
        a = ("gelu", "silu", "gelu_tanh", "relu6")[(i + len(group)) % 4]
        given, got = run(c, dtype, lambda r, q, name: torch.randn((r, q), generator=gen, device="cuda") * (q ** -0.5 if name in ("w", "wg", "wu") else 1.0), a)
        for name, (want, slack) in formulas(c.op, given, a).items():
            D.check(got[name], want, slack, "%s %s, %s" % (c.name, name, c.expect))


def test_the_device_gets_what_the_cases_are_for():
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the cases' words are for 148 SMs")
    for c in P.CASES:
        assert c.on_host(0) == c.on_host(148)


WITHOUT = {"linear": ["bias", "res", "z", "bias res z"], "gated": ["bg", "bu", "g", "u", "bg bu g u"],
           "linear_grad": ["dx", "dw", "db", "dz", "dx db", "dw dz", "dx dw", "dx dw db", "dx dw dz", "dx dw db dz"],
           "gated_grad": ["dx", "dwg", "dwu", "dbg", "dbu", "dx dwg", "dx dwu", "dwg dwu", "dwg dbg", "dwu dbu", "dx dwg dwu", "dx dwg dwu dbg", "dx dwg dwu dbg dbu"]}


@pytest.mark.parametrize("op", list(P.STRUCTS))
@pytest.mark.parametrize("size", [(5, 200, 104), (130, 72, 264), (1500, 264, 520), (7, 129, 33), (1100, 65, 43)], ids=str)
def test_what_is_left_out(size, op):
    """Every optional matrix and vector is null once: the others are what they are with it."""
    for without in WITHOUT[op]:
        for out_pad, pad in ((0, 0), (3, 1)):
            gen = torch.Generator(device="cuda").manual_seed(sum(size))
            c = P.Case("without " + without, op, *size, "", without, pad=pad, out_pad=out_pad)
            given, got = run(c, torch.bfloat16, lambda r, q, name: torch.randint(-2, 3, (r, q), generator=gen, device="cuda").float())
            for name, (want, _) in formulas(op, given, c.act).items():
                assert (name in got) == (name not in c.without)
                if name in got:
                    assert torch.equal(got[name], want.to(got[name].dtype)), (without, name, c.on_host(0))


@pytest.mark.parametrize("size", [(200, 136, 264), (3001, 40, 33), (90, 33, 57), (2500, 24, 130)], ids=str)
@pytest.mark.parametrize("place", ["dy", "z"])
def test_dz_in_the_place_of_an_input(size, place):
    """dz over dy or over z, in rows on the 16-byte boundaries and off them, wide strips and narrow ones."""
    m, k, n = size
    for pad in (0, 1):
        gen = torch.Generator(device="cuda").manual_seed(m)
        c = P.Case("", "linear_grad", m, k, n, "", pad=pad, out_pad=pad, act="relu")
        whole = lambda r, q: torch.randint(-2, 3, (r, q), generator=gen, device="cuda").float()
        mats = {t: Matrix(*s, GUARD if t in ("dx", "dw") else float("nan"), torch.float16) for t, s in c.matrices().items() if t != "dz"}
        for t in ("dy", "x", "w", "z"):
            mats[t].t.copy_(whole(*mats[t].t.shape))
        given, db = {t: mats[t].t.clone() for t in ("dy", "x", "w", "z")}, torch.zeros(n, device="cuda")
        mats["dz"] = mats[place]
        args = c.pack("f16", lambda t: db.data_ptr() if t == "db" else mats[t].t.data_ptr())
        need = C.c_size_t()
        B._check(B.lib().dlf_linear_grad_workspace_bytes(args, C.byref(need)), "")
        ws = torch.empty(max(1, need.value), device="cuda", dtype=torch.uint8)
        B._check(B.lib().dlf_linear_grad(args, ws.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream), "dlf_linear_grad")
        got = {"dx": mats["dx"].t, "dw": mats["dw"].t, "dz": mats["dz"].t, "db": db}
        for name, (want, _) in formulas("linear_grad", given, "relu").items():
            assert torch.equal(got[name], want.to(got[name].dtype)), (name, pad)
    dense.synchronize()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["float16", "bfloat16"])
@pytest.mark.parametrize("op", list(P.STRUCTS))
@pytest.mark.parametrize("size", [(1, 200000, 72), (40, 100000, 64), (100000, 64, 40), (70, 72, 100000), (33, 20001, 35), (20001, 35, 33), (35, 33, 20001)], ids=str)
def test_long_and_thin(size, op, dtype):
    """One size far above the others: sums of many terms, many strips, a single tile."""
    gen = torch.Generator(device="cuda").manual_seed(sum(size))
    c = P.Case(str(size), op, *size, "")
    given, got = run(c, dtype, lambda r, q, name: torch.randint(-2, 3, (r, q), generator=gen, device="cuda").float())
    for name, (want, _) in formulas(op, given, c.act).items():
        assert float(want.abs().max()) < 2 ** 24
        assert torch.equal(got[name], want.to(got[name].dtype)), (name, c.on_host(0))

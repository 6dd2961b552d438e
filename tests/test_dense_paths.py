"""Which kernel and layout a dense operator's call gets, asked of the host's estimates for 148 SMs: the cases of the device's tests reach what they
are there for, and between them everything."""
import ctypes as C

import pytest

from paper_2011_05630_b200 import binding as B
from tests import dense_paths as P


def test_every_case_gets_the_kernel_that_it_is_there_for():
    for c in P.CASES:
        assert c.expect in P.parts(c.on_host()), (c.name, c.expect, c.on_host())


def test_the_cases_reach_everything():
    reached = {part for c in P.CASES for part in P.parts(c.on_host())}
    assert not [r for r in P.REACHED if r not in reached]


def test_no_case_reaches_what_is_not_listed_without_a_name():
    """Kernels that the texts name are these five."""
    assert {part.split("(")[0] for c in P.CASES for part in P.parts(c.on_host())} == {"dense_gemv", "dense_lat", "dense_pair", "dense_grad", "dense_pack"}


def test_the_question_itself():
    f, c = B.lib().dlf_linear_kernels, P.Case("", "linear", 40, 64, 32, "")
    args = c.pack("bf16", {t: i + 1 << 30 for i, t in enumerate(P.ORDER["linear"].split())}.get)
    text = C.create_string_buffer(200)
    assert f(args, 148, None, 200) == B.E_INVALID_ARG and f(args, 148, text, 0) == B.E_INVALID_ARG
    assert f(args, -1, text, 200) == B.E_INVALID_ARG and f(None, 148, text, 200) == B.E_INVALID_ARG
    whole = c.on_host().encode()
    assert whole.startswith(b"dense_lat(") and len(whole) > 64
    for size in (1, 2, 10, 64):   # cut off where the room ends, with an end
        text = C.create_string_buffer(b"x" * 200, 200)
        assert f(args, 148, text, size) == B.OK
        assert text.raw == whole[:size - 1] + b"\0" + b"x" * (200 - size)
    assert P.Case("", "gated", 0, 64, 32, "").on_host() == "" and P.Case("", "gated_grad", 0, 64, 32, "").on_host() == ""
    assert P.Case("", "linear_grad", 40, 64, 32, "", without="dx dw dz z db", act="none").on_host() == ""   # nothing asked for
    with pytest.raises(B.DlfError) as e:
        P.Case("", "linear", 40, 0, 32, "").on_host()
    assert e.value.status == B.E_SHAPE


@pytest.mark.parametrize("op", list(P.STRUCTS))
def test_the_answer_goes_with_the_workspace(op):
    """Copies and a gradient of its own are what a workspace is for: a call that names a dense_pack wants one."""
    for c in P.CASES:
        if c.op != op:
            continue
        mats = c.matrices()
        at = {t: (i + 1 << 30) + 2 * (mats[t][3] if t in mats else 0) for i, t in enumerate(P.ORDER[op].split())}
        need = C.c_size_t()
        B._check(getattr(B.lib(), "dlf_%s_workspace_bytes" % op)(c.pack("bf16", at.get), C.byref(need)), op)
        names = [part.split("(")[0] for part in P.parts(c.on_host())]
        assert (need.value > 0) == ("dense_pack" in names or (op.endswith("grad") and not (op == "linear_grad" and (c.out_pad + c.n) % 8 == 0 and c.out_shift % 8 == 0))), c.name


@pytest.mark.parametrize("sms", [1, 2, 3, 20, 132, 148, 160])
def test_any_number_of_sms_has_an_answer(sms):
    for c in P.CASES:
        names = [part.split("(")[0] for part in P.parts(c.on_host(sms))]
        assert names and not set(names) - {"dense_gemv", "dense_lat", "dense_pair", "dense_grad", "dense_pack"}, (c.name, sms)

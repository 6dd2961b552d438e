"""Rules of the dense operators' sources that no run can show."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2011_05630_b200", "csrc")


def test_what_names_a_file_s_own_variable_is_a_file_s_own_function():
    """A header's `static` variable is another one in every source file: an inline function that names it would have several meanings, of which
    the linker keeps one.  So the host's functions that name such a variable, or one of these functions, are static, too."""
    seen = 0
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".h", ".cuh")):
            continue
        src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        own = set(re.findall(r"^static __device__ [\w ]+? (\w+)(?:\[\d*\])?(?: =[^;]*)?;", src, re.M))
        functions = re.findall(r"^([^\s{}#][^\n;={}]*?\b(\w+)\([^\n;]*\)) \{(.*?)^\}", src, re.M | re.S)
        while True:
            more = {f for _, f, body in functions for v in own if re.search(r"\b%s\b" % v, body)} - own
            if not more:
                break
            own |= more
        for head, f, _ in functions:
            if f in own:
                seen += 1
                assert re.search(r"\bstatic\b", head), (name, head)
    assert seen >= 1


def test_the_stall_s_arguments():
    from paper_2011_05630_b200 import binding as B
    for which, us in ((-1, 1000), (2, 1000), (0, 0), (1, -5), (0, 1000001)):
        assert B.lib().dlf_dense_debug_stall(which, us, None) == B.E_INVALID_ARG

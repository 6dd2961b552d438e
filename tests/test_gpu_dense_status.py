"""What dense.synchronize() tells of a wait that gave up: every thread, once, of either kernel, and nothing is lost to another's report."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

CODE = """
import threading
import torch
from paper_2011_05630_b200 import binding as B, dense

x, w = torch.ones((40, 64), device="cuda").half(), torch.ones((24, 64), device="cuda").half()


def told():
    try:
        dense.synchronize()
        return False
    except B.DlfError as e:
        assert e.status == B.E_TIMEOUT, e
        return True


class Other(threading.Thread):   # a thread that answers as often as it is asked
    def __init__(self):
        super().__init__(daemon=True)
        self.ask, self.done, self.answer = threading.Semaphore(0), threading.Semaphore(0), None
        self.start()

    def run(self):
        while True:
            self.ask.acquire()
            self.answer = told()
            self.done.release()

    def told(self):
        self.ask.release()
        assert self.done.acquire(timeout=60)
        return self.answer


other = Other()
assert not told() and not other.told()
for which in (0, 1):
    B._check(B.lib().dlf_dense_debug_stall(which, 1000, torch.cuda.current_stream().cuda_stream), "stall")   # (a millisecond)
    assert told() and not told()
    assert other.told() and not other.told()
    for i in (0, 1):   # both kernels: one report
        B._check(B.lib().dlf_dense_debug_stall(i, 1000, torch.cuda.current_stream().cuda_stream), "stall")
    assert other.told() and not other.told()
    assert told() and not told()
    assert bool((dense.linear(x, w) == 64).all())   # the context is intact
assert not told()
print("told")
"""


def test_every_thread_is_told_of_a_wait_that_gave_up():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CODE], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "told" in r.stdout, r.stderr[-2000:]

"""The largest lists in a thread with a small stack: the host side of hydra_grad_norm and hydra_grad_clip keeps what it
knows of up to 4096 tensors in some 16 KB.  In processes of their own, where an overflow would end the process, and with
no GPU visible, so that the calls that pass the checks end in the launch's error."""
import os
import subprocess
import sys

import pytest

import paper_2309_00754_amd as H

pytestmark = pytest.mark.skipif(not os.path.exists(H.LIB_PATH), reason="libhydra.so not built")

PROGRAM = """
import ctypes, sys, threading
import paper_2309_00754_amd as H
from paper_2309_00754_amd import _binding

L = H.lib()
n, at = 4096, 0x40000000
order = [(5 * i) % n for i in range(n)]                       # a permutation
g = (ctypes.c_void_p * n)(*[at + 4096 * i for i in order])
o = (ctypes.c_void_p * n)(*[at * 4 + 4096 * i for i in order])
types = (ctypes.c_int32 * n)(*[H.HYDRA_F32] * n)
numels = (ctypes.c_int64 * n)(*[1000] * n)
nbytes = H.hydra_grad_norm_workspace_bytes()
head = (n, g, types, numels)

def call(kind):
    norm, ws = 0x100000, 0x200000
    if kind == "norm":
        return L.hydra_grad_norm(*head, norm, ws, nbytes, None)
    if kind == "refused":
        return L.hydra_grad_clip(*head, 1.0, at + 4096 * (n - 1), None, None, ws, nbytes, None, None)
    if kind == "in place":
        return L.hydra_grad_clip(*head, 1.0, norm, None, None, ws, nbytes, None, None)
    return L.hydra_grad_clip(*head, 1.0, norm, o, types, ws, nbytes, None, None)

kind, got = sys.argv[1], []
first = call(kind)                                            # (the runtime sets itself up on the main thread)
threading.stack_size(64 << 10)
t = threading.Thread(target=lambda: got.append(call(kind)))
t.start()
t.join()
print(first, *got)
"""


@pytest.mark.parametrize("kind", ["refused", "norm", "in place", "into others"])
def test_largest_lists_in_a_small_stack(kind):
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1")
    r = subprocess.run([sys.executable, "-c", PROGRAM, kind], env=env, capture_output=True, text=True, timeout=120,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, f"exit status {r.returncode}\n{r.stderr[-2000:]}"
    code = H.HYDRA_ERR_SHAPE if kind == "refused" else H.HYDRA_ERR_HIP
    assert r.stdout.split() == [str(int(code))] * 2

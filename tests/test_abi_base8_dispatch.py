"""The most rows of blocks that one call of hydra_fp8_quantize takes: sixteen blocks of 128 values are a workgroup of 256
threads, and a launch counts its threads in 32 bits.  In processes of their own with no GPU visible, so that a call that
passes the checks ends in the launch's error."""
import os
import subprocess
import sys

import pytest

import paper_2309_00754_amd as H

pytestmark = pytest.mark.skipif(not os.path.exists(H.LIB_PATH), reason="libhydra.so not built")

PROGRAM = """
import sys
import paper_2309_00754_amd as H
M, K = int(sys.argv[1]), int(sys.argv[2])
print(H.lib().hydra_fp8_quantize(0x100000, H.HYDRA_BF16, M, K, 1, 0x200000, 0x300000, None, None, None))
"""


@pytest.mark.parametrize("M,blocks,code", [
    (65520, 4097, H.HYDRA_ERR_HIP),        # 2^28 - 16: as many as there may be
    (16385, 16383, H.HYDRA_ERR_SHAPE),     # 2^28 - 1
    (89478485, 3, H.HYDRA_ERR_SHAPE),      # (2^28 - 1 too, of more rows than a matrix may have)
    (1 << 15, 1 << 13, H.HYDRA_ERR_SHAPE),
])
@pytest.mark.parametrize("short", [0, 127])
def test_most_blocks_of_rows(M, blocks, code, short):
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1")
    r = subprocess.run([sys.executable, "-c", PROGRAM, str(M), str(blocks * 128 - short)], env=env, capture_output=True,
                       text=True, timeout=120, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.split() == [str(int(code))]

"""What hydra_fp8_lora_linear_backward asks its caller for is what its launches use, and no more: up to 512 rows dA and dB have
no partial sums, and the base product's lie where the outer products' come later.  Without a GPU."""
import os

import pytest

import paper_2309_00754_amd as H

pytestmark = pytest.mark.skipif(not os.path.exists(H.LIB_PATH), reason="libhydra.so not built")


def up(n, to=256):
    return -(-n // to) * to


def used(M, N, K, r):
    """dy's bytes and scales; B^T, A^T and s U of two bytes (s U four); three planes each of s U and s T; eight partial sums
    each of U and T; and the larger of the base product's partial sums (eight of dx, or 512 of 128 x 256) and the outer products'."""
    rp = 0 if r == 0 else max(16, 1 << (r - 1).bit_length())
    n = up(M * N) + up(M * -(-N // 128))
    n += up(2 * rp * N) + up(2 * rp * K) + up(4 * rp * M)
    n += 2 * up(6 * rp * up(M, 32)) + 2 * up(32 * rp * M)

    def outer(C):
        if M <= 512:
            return 0
        tiles = -(-C // 256)
        rows = max(64, up(-(-M // max(1, -(-256 // tiles))), 32))
        return up(-(-M // rows) * rp * C * 4)

    split = 0 if N <= 896 else up(4 * min(8 * M * K, 512 * 128 * 256))
    return n + max(split, outer(K) + outer(N))


@pytest.mark.parametrize("M,N,K,r", [(1, 16, 16, 1), (16, 4096, 4096, 16), (250, 8192, 2048, 128), (512, 11008, 4096, 64),
                                     (513, 4096, 4096, 16), (2048, 4096, 4096, 16), (2100, 688, 2048, 100),
                                     (3945, 8192, 864, 128), (300, 4096, 11008, 0)])
def test_the_backward_asks_for_what_it_uses(M, N, K, r):
    assert H.hydra_fp8_lora_linear_backward_workspace_bytes(M, N, K, r) <= used(M, N, K, r)

"""hydra_grad_clip into other tensors: the norm and the flag may not lie in a gradient, which the scaling still reads when
they are written.  Refused on the host before any HIP call: no GPU."""
import ctypes
import os

import pytest

import paper_2309_00754_amd as H

pytestmark = pytest.mark.skipif(not os.path.exists(H.LIB_PATH), reason="libhydra.so not built")

BF, F = H.HYDRA_BF16, H.HYDRA_F32


def at(i):
    return 0x100000 + 0x10000 * i  # fake device addresses, never dereferenced


def _clip(g, t, n, outs, ot, norm, err=None):
    k = len(g)
    return H.lib().hydra_grad_clip(k, (ctypes.c_void_p * k)(*g), (ctypes.c_int32 * k)(*t), (ctypes.c_int64 * k)(*n), 1.0,
                                   norm, (ctypes.c_void_p * k)(*outs), (ctypes.c_int32 * k)(*ot), at(30),
                                   H.hydra_grad_norm_workspace_bytes(), err, None)


# gradient 0: 64 fp32 (256 bytes), gradient 1: 100 bf16 (200 bytes)
INSIDE = [(0, 0), (0, 16), (0, 252), (1, 0), (1, 196)]


@pytest.mark.parametrize("which,off", INSIDE)
@pytest.mark.parametrize("outs", [(2, 3), (5, 4), (2, 1), (0, 3)])  # apart, in descending order, one of them in place
def test_norm_or_flag_inside_a_gradient_is_refused(which, off, outs):
    ot = (F, BF)
    head = ((at(0), at(1)), (F, BF), (64, 100), [at(o) for o in outs], ot)
    assert _clip(*head, norm=at(which) + off) == H.HYDRA_ERR_SHAPE
    assert _clip(*head, norm=at(8), err=at(which) + off) == H.HYDRA_ERR_SHAPE


def test_norm_or_flag_that_reaches_into_a_gradient_is_refused():
    """Four bytes that end two bytes into a bf16 gradient."""
    head = ((at(0), at(1) + 2), (F, BF), (64, 99), (at(2), at(3)), (F, BF))
    assert _clip(*head, norm=at(1)) == H.HYDRA_ERR_SHAPE
    assert _clip(*head, norm=at(8), err=at(1)) == H.HYDRA_ERR_SHAPE


def test_many_gradients_in_any_order():
    order = [(7 * i) % 300 for i in range(300)]
    g, outs = [0x40000000 + 4096 * i for i in order], [0x80000000 + 4096 * i for i in range(300)]
    head = (g, [F] * 300, [1000] * 300, outs, [F] * 300)
    for i in (0, 1, 150, 299):
        assert _clip(*head, norm=g[i] + 2000) == H.HYDRA_ERR_SHAPE
        assert _clip(*head, norm=at(8), err=g[i] + 3996) == H.HYDRA_ERR_SHAPE

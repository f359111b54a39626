"""The binding's checks of the update step's operators that need no GPU: tensors on the host are refused, and a call
whose tensors or stream are not all on one device never reaches the library."""
import os

import pytest
import torch

import paper_2309_00754_amd as H
from paper_2309_00754_amd import _binding as Bd

pytestmark = pytest.mark.skipif(not os.path.exists(H.LIB_PATH), reason="libhydra.so not built")


def test_host_tensors_are_refused():
    x, v = torch.zeros(2, 8), torch.zeros(2)
    with pytest.raises(ValueError):
        H.hydra_layer_norm(x, None, None, x.clone())
    with pytest.raises(ValueError):
        H.hydra_layer_norm_backward(x, x, None, v, v, x.clone())
    with pytest.raises(ValueError):
        H.hydra_token_logprobs(x, torch.zeros(2, dtype=torch.int32), v)
    with pytest.raises(ValueError):
        H.hydra_token_logprobs_backward(x, torch.zeros(2, dtype=torch.int32), v, x.clone(), v)
    with pytest.raises(ValueError):
        H.hydra_grad_norm([x], torch.zeros(1))
    with pytest.raises(ValueError):
        H.hydra_grad_clip([x], 1.0, torch.zeros(1))


class _On:
    """What _launch looks at of a tensor or a stream."""

    def __init__(self, device):
        self.device = torch.device(device)


def _never(*args):
    raise AssertionError("the library was called")


def test_tensors_on_two_devices_are_refused():
    with pytest.raises(ValueError, match="different devices"):
        Bd._launch("call", (_On("cuda:0"), None, _On("cuda:1")), None, _never)


def test_a_stream_of_another_device_is_refused():
    with pytest.raises(ValueError, match="stream belongs to cuda:0"):
        Bd._launch("call", (_On("cuda:1"), _On("cuda:1")), _On("cuda:0"), _never)


def test_rows_may_stand_apart_and_not_overlap(monkeypatch):
    class Gpu(torch.Tensor):
        device = torch.device("cuda:0")

    def on_gpu(t):
        return t.as_subclass(Gpu)

    z = torch.zeros(6, 20)
    assert Bd._rows(on_gpu(z), "z") == 20
    assert Bd._rows(on_gpu(z[:, :7]), "z") == 20
    assert Bd._rows(on_gpu(z[:1, :7]), "z") == 7
    assert Bd._rows(on_gpu(z[::2, 3:4]), "z") == 40
    for bad in (z.t(), z[:, ::2], z.view(-1).as_strided((4, 20), (10, 1)), z.view(-1), z[:1].expand(6, 20)):
        with pytest.raises(ValueError):
            Bd._rows(on_gpu(bad), "z")
    with pytest.raises(ValueError):
        Bd._rows(on_gpu(z), "z", (6, 21))
    with pytest.raises(TypeError):
        Bd._rows(on_gpu(z.double()), "z")

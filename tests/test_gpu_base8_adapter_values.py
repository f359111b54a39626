"""Values at the ends of the range in the adapter's own input of the linear over an 8-bit base, at ranks that are padded."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from gpu_helpers import say
from update_helpers import U, empty, f64, near, put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,r", [(3, 40, 128, 1), (40, 300, 256, 1), (1100, 264, 128, 1), (20, 64, 8192, 1)])
def test_the_largest_and_infinite_updates(dev, M, N, K, r):
    """An infinity in the adapter's own input makes its row's outputs infinite by the sign of B, a NaN makes them NaN, and
    numbers next to the largest stay what they are."""
    import torch
    say("largest and infinite updates", M, N, K)
    g = np.random.default_rng(M)
    xa = np.zeros((M, K), np.float32)
    xa[:, K - 1] = g.choice([-1, 1], M) * 2.0 ** 126 * (1 + np.arange(M) % 128 / 128)
    xa[0, K - 1], xa[1, K - 1], xa[2, K - 1] = np.inf, -np.inf, np.nan
    B = g.choice([-1.0, -0.75, 0.5, 1.0], (N, r))
    x, A = put(np.ones((M, K)), "bf16", dev), put(np.ones((r, K)), "bf16", dev)
    W, w = torch.zeros((N, K), dtype=torch.uint8, device=dev), torch.full((-(-N // 128), -(-K // 128)), 127, dtype=torch.uint8, device=dev)
    on = empty((M, N), "f32", dev)
    H.hydra_fp8_lora_linear(x, W, w, A, put(B, "bf16", dev), 1.9921875, None, on, x_adapter=put(xa, "bf16", dev))
    ref = 1.9921875 * xa[:, K - 1:].astype(np.float64) @ B.T
    near(f64(on), ref, 4 * U * np.abs(ref), "y_on")

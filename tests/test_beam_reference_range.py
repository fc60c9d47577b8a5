"""The plain implementation of beam selection where logits are very large or very low, against
PyTorch's log_softmax in 64 bits (CPU)."""
import numpy as np
import pytest
import torch

import _beam_reference as ref


@pytest.mark.parametrize("low", [-3.4028234663852886e38, -1e30, -1e12, -2e10, 2e10, 1e12, 1e30])
def test_scores_are_those_of_a_log_softmax(low):
    """Rows of one value (a dead beam masked by the type's lowest number), beside live ones, and with a larger one."""
    rng = np.random.default_rng(1)
    x = rng.normal(0, 2, (4, 50))
    x[1] = low
    x[2] = low
    x[2, 30:] = low / 2 if low < 0 else low * 2
    x[3, 7] = abs(low)
    s = np.array([-2.0, -9.0, -1.0, -4.0])
    got = ref.select(x, [0, 4], 200, s)
    lp = s[:, None] + torch.log_softmax(torch.from_numpy(x), 1).numpy()
    at = np.array(got["parent"][0]), np.array(got["token"][0])
    np.testing.assert_allclose(got["score"][0], lp[at], rtol=1e-14, atol=1e-12)
    # the dead beam's tokens are s - log n, not 0
    dead = [z for p, z in zip(got["parent"][0], got["score"][0]) if p == 1]
    np.testing.assert_allclose(dead, -9.0 - np.log(50), rtol=1e-14)

"""The plain implementations of beam selection and distillation where logits are very large, very
low or far apart, against PyTorch's log_softmax in 64 bits (CPU)."""
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


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("T,far", [(1.0, 720.0), (1.0, 1e4), (0.01, 15.0), (1.0, 3.4028234663852886e38)])
def test_teachers_far_below_their_best_keep_their_logarithm(reverse, T, far):
    """Tops up to far below the largest, one column named twice there, and a tail as far: log p in the log domain."""
    rng = np.random.default_rng(2)
    z = rng.normal(0, 1, (2, 12)) * T
    index = np.array([[3, 5, 7, 7, 9], [0, 1, 2, 3, 4]])
    t = np.array([[1.0, 0.5, -far, -far, 0.2], [2.0, 1.0, -far, 0.0, -far]])
    tail = np.array([0.3, -far / T if far < 1e30 else -far])
    loss, grad, _, _ = ref.distill(z, t, index, tail, None, T, reverse)
    for r in range(2):
        cols = sorted(set(index[r].tolist()))
        logs = [torch.logsumexp(torch.tensor([x / T for x, v in zip(t[r], index[r]) if v == c], dtype=torch.float64), 0)
                for c in cols] + [torch.tensor(tail[r], dtype=torch.float64)]
        lp = torch.log_softmax(torch.stack(logs), 0)
        leaf = torch.from_numpy(z[r]).requires_grad_()
        lq = torch.log_softmax(leaf / T, 0)
        rest = torch.logsumexp(lq[[c for c in range(12) if c not in cols]], 0)
        lq = torch.cat([lq[cols], rest[None]])
        terms = lq.exp() * (lq - lp) if reverse else torch.where(lp.exp() > 0, lp.exp() * (lp - lq), 0.0)
        want = T * T * terms.sum()
        np.testing.assert_allclose(loss[r], want.item(), rtol=1e-12)
        want.backward()
        np.testing.assert_allclose(grad[r], leaf.grad.numpy(), rtol=1e-10, atol=1e-12)

"""The plain implementations of beam selection, forked pages and distillation against
brute force, invariants, PyTorch's autograd in 64 bits and differences (CPU)."""
import itertools
import math

import numpy as np
import pytest
import torch

import _beam_reference as ref


@pytest.mark.parametrize("seed", range(6))
def test_selection_is_the_whole_ranking_cut(seed):
    rng = np.random.default_rng(seed)
    rows, cols, k = 7, 13, int(rng.integers(1, 30))
    x, s = np.round(rng.normal(0, 2, (rows, cols))), np.round(rng.normal(-3, 1, rows))   # ties
    x[rng.random((rows, cols)) < 0.3] = -math.inf
    off = [0, 3, 3, 7]
    got = ref.select(x, off, k, s, log_probs=True)
    for b in range(3):
        every = sorted((-(s[r] + x[r, v]), r, v) for r in range(off[b], off[b + 1]) for v in range(cols)
                       if x[r, v] > -math.inf)[:k]
        n = len(every)
        assert got["count"][b] == n
        assert list(zip(got["parent"][b], got["token"][b]))[:n] == [(r, v) for _, r, v in every]
        assert got["parent"][b][n:] == [-1] * (k - n)


def test_two_steps_of_selection_are_a_beam_search():
    """With as many beams as columns the second step's list is the ranking of all pairs."""
    rng = np.random.default_rng(1)
    V = 5
    first, then = torch.log_softmax(torch.from_numpy(rng.normal(0, 2, (1, V))), 1).numpy(), rng.normal(0, 2, (V, V))
    a = ref.select(first, [0, 1], V, paths=[[0, 0]], path_len=[0])
    order = a["token"][0]
    b = ref.select(then[order], [0, V], 6, score=a["score"][0], paths=a["paths"][0], path_len=a["path_len"][0])
    lp = torch.log_softmax(torch.from_numpy(then), 1).numpy()
    want = sorted((-(first[0, u] + lp[u, v]), u, v) for u, v in itertools.product(range(V), range(V)))[:6]
    assert b["paths"][0] == [[u, v] for _, u, v in want]
    np.testing.assert_allclose(b["score"][0], [-s for s, _, _ in want], rtol=1e-12)


@pytest.mark.parametrize("seed", range(40))
def test_forked_pages_keep_their_holders(seed):
    """After any fork every page is free, held by as many rows as its count says, or kept outside."""
    rng = np.random.default_rng(seed)
    B, page, most, pool = 6, 4, 5, 40
    table, shared = np.full((B, most), -1), np.zeros(pool, int)
    free, n_free = list(rng.permutation(pool)), pool
    held, texts = [0] * B, [[] for _ in range(B)]
    cache = {}
    pinned = []
    for step in range(12):
        src = rng.integers(-1, B, B)
        keep = [0 if s < 0 else int(rng.integers(0, held[s] + 1)) for s in src]
        f = ref.fork(held, keep, table, free, n_free, shared, page, src)
        new = [texts[s][:n] if s >= 0 else [] for s, n in zip(src, f["length"])]
        for a, b, n in zip(f["copy_src"], f["copy_dst"], f["copy_len"]):
            for t in range(n):
                cache[b, t] = cache[a, t]
        table = np.array([[-1 if p is None else p for p in r] for r in f["table"]])
        free, n_free, shared, held, texts = f["free"], f["n_free"], f["shared"], f["length"], new
        for j in range(B):                                   # grow the rows by a few tokens of their own
            for _ in range(int(rng.integers(0, 4))):
                if held[j] == most * page or (held[j] % page == 0 and n_free == 0):
                    break
                if held[j] % page == 0:
                    n_free -= 1
                    table[j, held[j] // page] = free[n_free]
                    free[n_free] = None
                cache[table[j, held[j] // page], held[j] % page] = (step, j, held[j])
                texts[j].append((step, j, held[j]))
                held[j] += 1
        holders = np.zeros(pool, int)
        for j in range(B):
            for p in table[j, :-(-held[j] // page)]:
                holders[p] += 1
            assert [cache[table[j, t // page], t % page] for t in range(held[j])] == texts[j]
        for p in pinned:
            holders[p] += 1
        live = [p for p in range(pool) if holders[p]]
        assert sorted(free[:n_free]) == [p for p in range(pool) if not holders[p]]
        assert [shared[p] for p in live] == [holders[p] - 1 for p in live]
        if step == 3 and live:                               # the caller keeps a page for itself
            pinned.append(live[0])
            shared[live[0]] += 1


def torch_distill(z, teacher, index, tail, weight, T, reverse):
    """The definition in torch, float64."""
    total = []
    for r in range(z.shape[0]):
        cols = sorted({int(v) for v in index[r] if 0 <= v < z.shape[1]})
        t = [torch.logsumexp(torch.tensor([float(x) / T for x, v in zip(teacher[r], index[r]) if v == c]), 0) for c in cols]
        lp = torch.log_softmax(torch.stack([x.double() for x in t] + [torch.tensor(float(tail[r])).double()]), 0)
        lq = torch.log_softmax(z[r] / T, 0)
        out = torch.ones(z.shape[1], dtype=torch.bool)
        out[cols] = False
        lq = torch.cat([lq[cols], torch.logsumexp(lq[out], 0, keepdim=True)])
        far = (lq.exp() * (lq - lp)).sum() if reverse else (lp.exp() * (lp - lq)).sum()
        total.append(weight[r] * T * T * far)
    return torch.stack(total)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("T", [1.0, 0.5, 3.0])
def test_distillation_and_its_gradient(T, reverse):
    rng = np.random.default_rng(int(10 * T) + reverse)
    n, V, m = 5, 40, 6
    z, teacher = rng.normal(0, 2, (n, V)), np.float32(rng.normal(1, 2, (n, m))).astype(np.float64)
    index = np.stack([rng.permutation(V)[:m] for _ in range(n)])
    index[1, 3] = index[1, 0]                                # a column named twice
    index[2, 4:] = -1
    tail, weight = rng.normal(0, 1, n), rng.uniform(0.3, 2, n)
    loss, grad, _, _ = ref.distill(z, teacher, index, tail, weight, T, reverse)
    leaf = torch.from_numpy(z).requires_grad_()
    want = torch_distill(leaf, teacher, index, tail, weight, T, reverse)
    np.testing.assert_allclose(loss, want.detach().numpy(), rtol=1e-6)     # tails pass through fp32 in torch.tensor
    want.sum().backward()
    np.testing.assert_allclose(grad, leaf.grad.numpy(), rtol=1e-5, atol=1e-7)
    h = 1e-5
    for r, v in itertools.product(range(n), [0, 7, int(index[0, 0]), int(index[1, 0])]):
        up, down = z.copy(), z.copy()
        up[r, v] += h
        down[r, v] -= h
        a, b = (ref.distill(x, teacher, index, tail, weight, T, reverse)[0][r] for x in (up, down))
        assert abs((a - b) / (2 * h) - grad[r, v]) < 1e-8 + 1e-6 * abs(grad[r, v])


def test_distillation_without_a_tail_is_the_kl_of_the_renormalised_tops():
    rng = np.random.default_rng(5)
    z, t = rng.normal(0, 1, (3, 20)), rng.normal(0, 1, (3, 4))
    index = np.stack([rng.permutation(20)[:4] for _ in range(3)])
    loss, grad, _, _ = ref.distill(z, t, index)
    p, lq = torch.softmax(torch.from_numpy(t), 1), torch.log_softmax(torch.from_numpy(z), 1)
    want = (p * (p.log() - torch.gather(lq, 1, torch.from_numpy(index)))).sum(1)
    np.testing.assert_allclose(loss, want.numpy(), rtol=1e-12)
    full = torch.zeros(3, 20, dtype=torch.float64).scatter(1, torch.from_numpy(index), p)
    np.testing.assert_allclose(grad, (lq.exp() - full).numpy(), atol=1e-12)

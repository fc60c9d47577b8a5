"""Beam selection of rows whose logits are very large, very low or far apart, against PyTorch's
log_softmax in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2410_05165_amd.binding import AtspeedError  # noqa: E402
from paper_2410_05165_amd.paged import atspeed_beam_select  # noqa: E402

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def check(logits, off, k, score):
    """Scores are one rounding to fp32, a 64-bit sum of three numbers, and the logarithm of a sum of exponentials that
    are off by 2.4e-10 each; candidates further apart than that rank as they do in 64 bits."""
    got = atspeed_beam_select(logits, ints(off), k, score=score)
    lp = torch.log_softmax(logits.double().cpu(), 1).numpy() + score.double().cpu().numpy()[:, None]
    for b in range(len(off) - 1):
        every = sorted((-lp[r, v], r, v) for r in range(off[b], off[b + 1]) for v in range(lp.shape[1]) if lp[r, v] > -math.inf)
        want = every[:k]
        n = int(got.count[b])
        assert n == len(want)
        score_of = got.score[b, :n].double().cpu().numpy()
        exact = np.array([-z for z, _, _ in want])
        room = 2.0 ** -24 * np.abs(exact) + 2.0 ** -51 * np.abs(exact) + 2.5e-10
        assert (np.abs(score_of - exact) <= room).all(), (b, score_of[:5], exact[:5])
        parent, token = got.parent[b, :n].tolist(), got.token[b, :n].tolist()
        assert [(p, t) for p, t in zip(parent, token)] == [(r, v) for _, r, v in want]
    return got


LOWS = [("min", None), ("-1e30", -1e30), ("-1e20", -1e20), ("-1e12", -1e12)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [7, 1000, 1024, 1500, 33024])
@pytest.mark.parametrize("name,low", LOWS)
def test_a_beam_without_an_allowed_token_ranks_by_its_score(dtype, cols, name, low):
    """All of a row's logits the mask's number: each token has the score less log n, behind the live beams' tokens."""
    rng = np.random.default_rng(cols)
    low = torch.finfo(dtype).min if low is None else low
    x = torch.from_numpy(rng.normal(0, 1, (5, cols))).float().to(dtype)
    x[1] = low
    x[2, 3:] = low                                         # three tokens left
    x[4] = low
    score = torch.tensor([-1.0, -9.0, -2.0, -4.0, -3.0], device=DEV)
    got = check(x.to(DEV), [0, 3, 5], min(12, 2 * cols), score)
    assert got.parent[0, 0].item() in (0, 2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [5, 900, 1024, 1500, 2048, 33024])
@pytest.mark.parametrize("top", [2.0 ** 35, -2.0 ** 35, 1e12, -1e12, 1e20, 1.5e10, -1.5e10])
@pytest.mark.parametrize("others", ["far", "-infinity"])
def test_columns_far_below_a_large_logit_add_nothing(dtype, cols, top, others):
    """One logit, or a few, of very large magnitude: what lies far below them, columns behind a tile's end and masked
    ones among it, is no part of the row's sum."""
    x = torch.full((3, cols), -math.inf if others == "-infinity" else min(2 * top, -1.0) if top < 0 else 0.0).to(dtype)
    x[0, cols // 2] = top
    x[1, ::3] = top
    x[2] = top
    score = torch.tensor([-1.0, -2.5, -0.5], device=DEV)
    check(x.to(DEV), [0, 1, 3], 6, score)


@pytest.mark.parametrize("rows,cols", [(4104, 33024), (4104, 17000), (4104, 2048), (5400, 9000), (8196, 3000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_equal_rows_on_both_sides_of_the_cut_go_to_the_lower_one(rows, cols, dtype):
    """Rows that fill the card go to a wave each, those behind them in parts (4,096 or 8,192 come first), and the sums of
    the two differ in their last bits: no request has rows of both sorts, and its rows that are alike rank in order."""
    rng = np.random.default_rng(cols)
    whole, k, n = rows // 4096 * 4096, 24, 6 if rows < 6000 else 12
    off = np.arange(0, rows + 1, n)
    across = int(np.searchsorted(off, whole, "right")) - 1
    assert off[-1] == rows and off[across] < whole < off[across] + n
    x = torch.empty((rows, cols), dtype=dtype, device=DEV)
    for _ in range(3):
        x[:] = torch.from_numpy(rng.normal(0, 3, cols)).float().to(dtype).to(DEV)
        got = atspeed_beam_select(x, ints(off), k)
        best = torch.sort(x[0].float(), descending=True, stable=True)
        z, col = best.values[:k].tolist(), best.indices[:k].tolist()
        want = [(r, v) for _, r, v in sorted((-a, r, v) for a, v in zip(z, col) for r in range(n))][:k]
        for b in (0, across - 1, across, across + 1):
            if b >= len(off) - 1:
                continue
            assert [(p - int(off[b]), t) for p, t in zip(got.parent[b].tolist(), got.token[b].tolist())] == want, b
            assert bool((got.score[b] - got.score[0]).abs().max() <= 2.0 ** -23 * got.score[0].abs().max())


def test_paths_of_no_beams():
    """Empty paths: every parent is unknown and has an empty one; without rows there is nothing but padding."""
    x = torch.randn((4, 60), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    none, length = ints(np.zeros((0, 3))), ints([])
    for _ in range(3):
        torch.full((1 << 16,), 77, dtype=torch.int32, device=DEV)      # what fresh memory may hold
        got = atspeed_beam_select(x, ints([0, 3, 4]), 5, paths=none, path_len=length)
        assert torch.equal(got.paths[..., 0], got.token) and bool((got.paths[..., 1:] == -1).all())
        assert bool((got.path_len == 1).all())
        got = atspeed_beam_select(x[:0], ints([0, 0]), 2, paths=none, path_len=length)
        assert got.count.tolist() == [0] and bool((got.paths == -1).all()) and not bool(got.path_len.any())
    with pytest.raises(ValueError, match="max_path"):
        atspeed_beam_select(x, ints([0, 4]), 5, paths=ints(np.zeros((4, 0))), path_len=ints(np.zeros(4)))


def test_paths_of_no_beams_in_a_graph():
    x = torch.randn((4, 60), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    none, length, off = ints(np.zeros((0, 3))), ints([]), ints([0, 3, 4])
    want = atspeed_beam_select(x, off, 5, paths=none, path_len=length)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = atspeed_beam_select(x, off, 5, paths=none, path_len=length)
    for _ in range(3):
        for t in got:
            t.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        torch.full((1 << 16,), 77, dtype=torch.int32, device=DEV)


def test_paths_too_wide_are_refused_without_room_for_them():
    x = torch.randn((4, 60), device=DEV)
    for most in (1 << 30, (1 << 31) - 1):
        with pytest.raises(AtspeedError, match="max_path"):
            atspeed_beam_select(x, ints([0, 4]), 5, paths=ints(np.zeros((0, 1))).expand(0, most), path_len=ints([]))


@pytest.mark.parametrize("what", ["one", "wide", "empty", "short"])
def test_every_place_of_the_cut_among_the_requests(what):
    """The cut inside the last request, inside one of hundreds of rows, between empty ones, behind the rows that are used:
    every request has the ranking that it has by itself."""
    rng = np.random.default_rng(3)
    rows, cols, k = 4200, 2500, 7
    counts = {"one": [6] * 682 + [108], "wide": [1] * 3800 + [400], "empty": [0, 6] * 700, "short": [4] * 1023}[what]
    if what == "wide":
        counts = [5] * 760 + [400]
    off = np.concatenate([[0], np.cumsum(counts)])
    if what == "empty":
        off = np.concatenate([off[:1000], [4200]])
    x = torch.randn((rows, cols), generator=torch.Generator(device=DEV).manual_seed(4), device=DEV).to(BF16)
    score = torch.from_numpy(-rng.gamma(4, 2, rows)).float().to(DEV)
    got = atspeed_beam_select(x, ints(off), k, score=score)
    for b in {0, len(off) - 2, len(off) // 2} | {int(np.searchsorted(off, 4096, "right")) + d for d in (-3, -2, -1, 0)}:
        if not 0 <= b < len(off) - 1:
            continue
        r0, r1 = int(off[b]), int(off[b + 1])
        alone = atspeed_beam_select(x[r0:r1], ints([0, r1 - r0]), k, score=score[r0:r1].contiguous())
        n = int(alone.count[0])
        assert int(got.count[b]) == n == min(k, (r1 - r0) * cols)
        assert (got.parent[b, :n] - r0).tolist() == alone.parent[0, :n].tolist()
        assert got.token[b].tolist() == alone.token[0].tolist()
        torch.testing.assert_close(got.score[b, :n], alone.score[0, :n], rtol=2.0 ** -23, atol=0)

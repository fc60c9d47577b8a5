"""Beam selection against its plain implementation in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import _beam_reference as ref  # noqa: E402
from paper_2410_05165_amd.binding import AtspeedError  # noqa: E402
from paper_2410_05165_amd.paged import atspeed_beam_select  # noqa: E402

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def floats(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV)


def case(seed, counts, cols, k, dtype=F32, masked=0.0, done=0.0, log_probs=False, path=0, base=0, spread=3.0, offset=0,
         stride=None, ids=True):
    """The call's arguments; logits are a piece of a larger tensor where offset or stride say so."""
    rng = np.random.default_rng(seed)
    rows, off = int(np.sum(counts)), np.concatenate([[0], np.cumsum(counts)])
    stride = cols if stride is None else stride
    whole = torch.full((offset + max(rows, 1) * stride + 64,), 50.0, dtype=dtype, device=DEV)    # would win if it were read
    logits = torch.as_strided(whole, (rows, cols), (stride, 1), offset)
    x = rng.normal(0, spread, (rows, cols))
    x[rng.random((rows, cols)) < masked] = -math.inf
    logits.copy_(floats(x).to(dtype))
    c = dict(logits=logits, row_off=off, k=k, score=np.float32(-rng.gamma(4, 2, rows)), token_base=base, log_probs=log_probs)
    if done:
        c["done"] = (rng.random(rows) < done).astype(np.int32)
    if ids:
        c["row_id"] = rng.permutation(rows)
    if path:
        c["paths"], c["path_len"] = rng.integers(0, 1000, (max(rows, 1), path)), rng.integers(-1, path + 2, max(rows, 1))
    return c


def run(c):
    on = dict(c)
    for name in ("row_off", "done", "row_id", "paths", "path_len"):
        if on.get(name) is not None:
            on[name] = ints(on[name])
    if on.get("score") is not None:
        on["score"] = floats(on["score"])
    return atspeed_beam_select(**on)


def check(c, got=None):
    got = run(c) if got is None else got
    want = ref.select(c["logits"].double().cpu().numpy(), c["row_off"], c["k"], c.get("score"), c.get("done"),
                      c.get("token_base", 0), c.get("log_probs", False), c.get("row_id"), c.get("paths"), c.get("path_len"))
    for name in ("count", "parent", "token") + (("paths", "path_len") if c.get("paths") is not None else ()):
        g = getattr(got, name).cpu().tolist()
        assert g == want[name], (name, [(i, a, b) for i, (a, b) in enumerate(zip(g, want[name])) if a != b][:3])
    score, w = got.score.double().cpu().numpy(), np.array(want["score"])
    live = np.isfinite(w)
    assert (np.isneginf(score) == ~live).all()
    # one rounding to fp32, and the logarithm of a sum of exponentials that are off by 2.4e-10 each
    assert (np.abs(score[live] - w[live]) <= 2.0 ** -24 * np.abs(w[live]) + 2.5e-10).all()
    return got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1, 2, 63, 64, 65, 500, 1023, 1024, 1025, 4096, 4099, 33024, 131073])
@pytest.mark.parametrize("k", [1, 10, 64])
def test_columns(dtype, cols, k):
    check(case(cols + k, [3, 1, 0, 5], cols, k, dtype, path=5, base=100))


@pytest.mark.parametrize("k", [1, 2, 63, 64, 65, 128, 191, 192, 193, 255, 256])
@pytest.mark.parametrize("counts,cols", [([1], 700), ([4, 2], 5000), ([9], 300), ([40, 1, 70], 129)])
def test_list_lengths(k, counts, cols):
    check(case(k, counts, cols, k, BF16 if k % 2 else F32))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("masked", [0.5, 0.97, 0.9999, 1.0])
@pytest.mark.parametrize("cols", [300, 9000])
def test_masked_columns_and_short_lists(dtype, masked, cols):
    check(case(int(100 * masked) + cols, [4, 1, 7], cols, 30, dtype, masked=masked, done=0.3, path=3))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("log_probs", [False, True])
def test_scores_of_log_probabilities(dtype, log_probs):
    check(case(3, [5, 8, 2], 2500, 20, dtype, masked=0.2, done=0.2, log_probs=log_probs, path=6))


@pytest.mark.parametrize("cols", [200, 5000, 20000])
@pytest.mark.parametrize("k", [1, 50, 200])
def test_equal_logits_go_to_the_lowest_columns(cols, k):
    """Rows of one value, of a few values, and of values that rise, fall and repeat."""
    c = case(cols + k, [6], cols, k, F32, ids=False)
    v = torch.arange(cols, device=DEV)
    for r, row in enumerate([0 * v, -0.0 * v, v % 3, (v // 64) % 5, -(v % 7), v * 0 - 2]):
        c["logits"][r] = row.float()
    c["logits"][1, ::2] = -0.0                             # equal to 0
    for s in (np.float32([0, 0, -1, -1, -2, -2]), np.float32([-9, -9, -9, 0, -9, -9]), None):
        check(dict(c, score=s))


def test_rows_that_are_alike_go_to_the_lowest_row():
    c = case(5, [7, 7], 3000, 40, BF16, ids=False)
    c["logits"][:] = c["logits"][:1].clone()
    c["score"][:] = -1.5
    got = check(c)
    assert got.parent[0, :7].tolist() == list(range(7)) and len(set(got.token[0, :7].tolist())) == 1


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("log_probs", [False, True])
@pytest.mark.parametrize("cols", [100, 6000])
def test_rows_without_a_distribution_have_no_candidates(dtype, log_probs, cols):
    c = case(cols, [9, 2], cols, 25, dtype, masked=0.1, log_probs=log_probs)
    x = c["logits"]
    for r, bad in enumerate([math.nan, -math.nan, math.inf]):
        x[r, (37 * r + 5) % cols] = bad
        x[r + 3, cols - 1 - r] = bad
    x[2, 3] = math.nan                                       # NaN and infinity together
    x[9] = -math.inf
    x[10] = math.nan
    c["score"][6], c["score"][7] = math.nan, -math.inf
    got = check(c)
    assert int(got.count[1]) == 0 and set(got.parent[0].tolist()) <= {int(c["row_id"][8]), -1}


def test_the_lowest_number_is_a_logit_like_others():
    for dtype in (F32, BF16):
        c = case(8, [2, 1], 1500, 12, dtype)
        low = torch.finfo(dtype).min
        c["logits"][:] = low
        c["logits"][0, 77] = 1.0
        c["logits"][2, 1400:] = low / 2
        check(c)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("spread", [1e-3, 30.0, 1e4])
def test_flat_and_steep_rows(dtype, spread):
    check(case(int(spread), [6, 6], 4000, 33, dtype, spread=spread))


def test_ended_beams_stay_as_they_are():
    c = case(4, [5, 3, 2], 800, 9, F32, path=4)
    c["done"] = np.array([1, 0, 1, 0, 0, 1, 1, 1, 0, 1])
    c["score"][2] = 3.0
    c["logits"][0] = math.nan                                # not read
    c["logits"][2] = math.inf
    got = check(c)
    first = int(c["row_id"][2])
    assert got.parent[0, 0] == first and got.token[0, 0] == -1 and got.score[0, 0] == 3.0
    assert got.path_len[0, 0] == min(max(c["path_len"][first], 0), 4)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,stride", [(0, 1031), (1, 1030), (3, 1037), (8, 2048)])
def test_rows_anywhere(dtype, offset, stride):
    check(case(offset, [4, 4], 1030, 16, dtype, offset=offset, stride=stride))


@pytest.mark.parametrize("counts,cols,k", [([300], 40, 200), ([1500, 3], 70, 50), ([1] * 1024, 90, 3), ([2600], 33, 256)])
def test_many_rows(counts, cols, k):
    check(case(len(counts), counts, cols, k, F32, masked=0.3))


@pytest.mark.parametrize("counts,cols,k,log_probs", [([7] * 600, 2100, 10, False), ([7] * 600, 2100, 70, True), ([9] * 456 + [1] * 3, 1500, 5, False),
                                                     ([4] * 1024, 1100, 4, False), ([4100], 1100, 20, False)])
def test_more_rows_than_waves_on_the_card(counts, cols, k, log_probs):
    """4,096 rows go to a wave each, those behind them in parts; one request has rows of both sorts."""
    check(case(cols + k, counts, cols, k, BF16, done=0.05, log_probs=log_probs, path=3))


def test_without_scores_and_names():
    c = case(6, [3, 2], 400, 7, F32, ids=False, path=2)
    check(dict(c, score=None))


def test_parents_outside_the_paths_have_empty_ones():
    c = case(6, [3, 3], 400, 7, F32, path=3)
    c["row_id"] = np.array([0, -5, 99, 1, 2 ** 31 - 1, 5])
    check(c)


def test_row_offsets_that_are_out_of_order_stay_inside():
    c = case(7, [3, 3, 3], 5000, 7, F32)
    for off in ([0, 9, 4, 6], [-5, 2, 2 ** 31 - 1, 9], [5, 3, 1, -1], [0, 3, 6, 2 ** 31 - 1]):
        got = run(dict(c, row_off=np.array(off)))
        torch.cuda.synchronize()
        ok = (got.parent >= -1) & (got.parent < 9) & (got.token >= -1) & (got.token < 5000)
        assert bool(ok.all())


def test_rows_past_the_last_request_are_left_out():
    c = case(9, [3, 2], 300, 5, F32, ids=False)
    more = torch.full((9, 300), 40.0, device=DEV)
    more[:5] = c["logits"]
    c["logits"], c["score"] = more, np.concatenate([c["score"], np.zeros(4, np.float32)])
    check(c)
    none = run(dict(c, logits=more[:0], score=None, row_off=np.zeros(3)))
    assert none.count.tolist() == [0, 0] and bool((none.parent == -1).all())


@pytest.mark.parametrize("k", [3, 40, 130])
@pytest.mark.parametrize("rows", [1, 70])
def test_lists_that_need_several_rounds(k, rows):
    """One beam has every candidate, far down in its parts' lists; the others have the next best heads."""
    c = case(k + rows, [rows, 2], 20000, k, F32, ids=False)
    c["logits"][0] = torch.linspace(3, 3.001, 20000, device=DEV)
    c["score"][:] = -1.5
    c["score"][0] = 4.0
    check(c)
    c["logits"][0, :2000] = 5.0                                # the first parts have equal ones
    check(c)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1024, 1025, 3000])
def test_rising_and_falling_rows(dtype, cols):
    """Every tile is better, or worse, than all before it: the pool is cut again and again, or never."""
    c = case(cols, [4], cols, 30, dtype, ids=False)
    v = torch.arange(cols, device=DEV).float()
    c["logits"][0], c["logits"][1] = v / 64, -v / 64
    c["logits"][2], c["logits"][3] = (v // 300) / 8, -(v // 300) / 8
    check(c)
    for k in (64, 65, 192, 193, 256):
        check(dict(c, k=k))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k", [20, 55, 56, 57, 64, 103, 104, 105, 160, 256])
def test_pools_that_overflow_within_a_tile(dtype, k):
    """More columns pass a bound than there is room for: flat rows, few levels (equal logits everywhere), and few columns left."""
    c = case(k, [3, 4], 7000, k, dtype, ids=False)
    check(c)
    g = torch.Generator(device=DEV).manual_seed(k)
    c["logits"][1] = torch.randint(0, 3, (7000,), generator=g, device=DEV).to(dtype)
    c["logits"][2] = 0.5
    c["logits"][3] = torch.randint(0, 200, (7000,), generator=g, device=DEV).to(dtype) / 16
    c["logits"][4, 300:6900] = -math.inf
    c["logits"][5, 1024:2048] = c["logits"][5, :1024]          # the second tile again holds what the first one had
    c["logits"][6] = torch.randn(7000, generator=g, device=DEV).to(dtype) - (torch.arange(7000, device=DEV) < 1024) * 8.0
    check(c)


def test_scores_whose_order_hangs_on_the_last_bits():
    """Beams of one distribution whose scores differ by one step of fp32: their candidates alternate in that order."""
    c = case(31, [6], 500, 60, F32, ids=False)
    c["logits"][:] = c["logits"][:1].clone()
    for i in range(1, 6):
        c["score"][i] = np.nextafter(c["score"][i - 1], np.float32(0), dtype=np.float32)
    got = check(c)
    assert got.parent[0, :6].tolist() == [5, 4, 3, 2, 1, 0]


def test_offsets_past_32_bits():
    """Rows whose first element lies past 2^31 and 2^32 elements."""
    stride = (1 << 31) + 8
    whole = torch.empty(2 * stride + 600, dtype=BF16, device=DEV)
    logits = torch.as_strided(whole, (3, 600), (stride, 1))
    logits.copy_(torch.randn((3, 600), device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)))
    check(dict(logits=logits, row_off=[0, 3], k=20, score=np.float32([-1, -1, -1])))


def test_repeats_bit_for_bit_on_streams_and_in_graphs():
    """Two calls that alternate on two streams and in two graphs equal their eager results."""
    cases = [case(20 + i, [5, 9, 1] if i else [5, 9], 9000 + i, 12 if i else 200, BF16, done=0.1, path=4) for i in range(2)]
    held = [dict(c, **{n: ints(c[n]) for n in ("row_off", "done", "row_id", "paths", "path_len")}, score=floats(c["score"]))
            for c in cases]
    want = [check(c) for c in cases]
    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))  # noqa: E731
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(device=DEV) for _ in cases], []
    for _ in range(5):
        for i, c in enumerate(held):
            with torch.cuda.stream(streams[i]):
                got.append((i, atspeed_beam_select(**c)))
    torch.cuda.synchronize()
    assert all(same(g, want[i]) for i, g in got)
    graphs, outs = [torch.cuda.CUDAGraph() for _ in cases], []
    for g, c in zip(graphs, held):
        with torch.cuda.graph(g):
            outs.append(atspeed_beam_select(**c))
    for _ in range(3):
        for g, o, w in zip(graphs, outs, want):
            for t in o:
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert same(o, w)


def test_refusals():
    x, off = torch.zeros((4, 50), device=DEV), ints([0, 4])
    atspeed_beam_select(x, off, 3)
    for kw in (dict(k=0), dict(logits=x.half()), dict(logits=x.t()), dict(row_off=off.long()), dict(row_off=off[:0]),
               dict(score=torch.zeros(3, device=DEV)), dict(score=torch.zeros(4, device=DEV).double()),
               dict(done=torch.zeros(4, dtype=torch.bool, device=DEV)), dict(row_id=ints([0, 1, 2])),
               dict(paths=ints([0, 1])), dict(paths=ints([[0, 1]]), path_len=ints([0, 1])), dict(row_off=off.cpu()),
               dict(paths=ints([[0, 1]])), dict(path_len=ints([])), dict(row_off=off[:1])):
        with pytest.raises(ValueError):
            atspeed_beam_select(**{**dict(logits=x, row_off=off, k=3), **kw})
    with pytest.raises(AtspeedError):
        atspeed_beam_select(x, off, 257)

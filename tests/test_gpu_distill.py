"""Distillation from top logits, loss and gradient, against the definition in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import _beam_reference as ref  # noqa: E402
from paper_2410_05165_amd.align import atspeed_distill_grad, atspeed_distill_loss, distill  # noqa: E402
from paper_2410_05165_amd.binding import AtspeedError  # noqa: E402

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
FORMS = [(False, False), (True, False), (True, True)]        # tail, reverse


def case(seed, rows, cols, m, dtype=F32, tail=True, reverse=False, T=1.0, spread=2.0, weight=True, offset=0, stride=None):
    rng = np.random.default_rng(seed)
    stride = cols if stride is None else stride
    whole = torch.full((offset + rows * stride + 64,), 60.0, dtype=dtype, device=DEV)
    logits = torch.as_strided(whole, (rows, cols), (stride, 1), offset)
    on = lambda a, t=F32: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV).to(t)  # noqa: E731
    logits.copy_(on(rng.normal(0, spread, (rows, cols))))
    teacher = on(rng.normal(3, spread, (rows, m)), dtype)
    index = np.stack([rng.permutation(cols)[:m] if cols >= m else rng.integers(0, cols, m) for _ in range(rows)])
    index[rng.random(index.shape) < 0.1] = -1
    if m > 4:
        index[::2, 3] = index[::2, 0]                          # a column named twice
    lse = torch.logsumexp(teacher.float() / T, 1)
    return dict(logits=logits, teacher_logit=teacher,
                teacher_index=torch.from_numpy(index.astype(np.int32)).to(DEV),
                tail=lse + on(rng.normal(-1.5, 1, rows)) if tail else None,
                weight=on(rng.uniform(0.2, 2, rows)) if weight else None, temperature=T, reverse=reverse)


def num(t):
    return None if t is None else t.double().cpu().numpy()


def check(c, grad_loss=None):
    loss, saved = atspeed_distill_loss(**c)
    grad = atspeed_distill_grad(c["logits"], c["teacher_index"], saved, grad_loss, c["temperature"])
    want, slope, off, slope_off = ref.distill(num(c["logits"]), num(c["teacher_logit"]), num(c["teacher_index"]).astype(int),
                                              num(c["tail"]), num(c["weight"]), float(np.float32(c["temperature"])),
                                              c["reverse"], num(grad_loss))          # the call takes the number as fp32
    got = num(loss)
    assert grad.dtype == c["logits"].dtype and grad.shape == c["logits"].shape
    fine = np.isfinite(want)
    assert (got[~fine] == want[~fine]).all()
    assert (np.abs(got[fine] - want[fine]) <= off[fine] + 1e-38).all()
    half = 2.0 ** -8 if grad.dtype == BF16 else 2.0 ** -24
    g = num(grad)
    # fp32 numbers below 2^-126 may be flushed, also on the way
    over = np.abs(g - slope) - (slope_off * (1 + half) + half * np.abs(slope) + 1e-36)
    assert not (over > 0).any(), (np.max(over), np.argwhere(over > 0)[:4].tolist())
    assert not np.isnan(g[~np.isnan(slope)]).any()
    return loss, grad


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tail,reverse", FORMS)
@pytest.mark.parametrize("cols,m", [(1, 1), (2, 1), (7, 7), (31, 5), (64, 64), (500, 10), (1024, 256), (4095, 32), (4097, 100),
                                    (33024, 64), (131073, 20)])
def test_sizes(dtype, tail, reverse, cols, m):
    check(case(cols + m, 6, cols, m, dtype, tail, reverse), torch.rand(6, device=DEV) + 0.5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tail,reverse", FORMS)
@pytest.mark.parametrize("T", [0.25, 0.7, 4.0])
@pytest.mark.parametrize("spread", [0.1, 8.0])
def test_temperatures(dtype, tail, reverse, T, spread):
    check(case(int(10 * T), 9, 777, 12, dtype, tail, reverse, T, spread))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tail,reverse", FORMS)
@pytest.mark.parametrize("offset,stride", [(0, 1003), (1, 1000), (5, 1009), (8, 1024)])
def test_rows_anywhere(dtype, tail, reverse, offset, stride):
    c = case(offset, 5, 1000, 9, dtype, tail, reverse, offset=offset, stride=stride, weight=False)
    _, grad = check(c)
    whole = torch.full((offset + 5 * stride + 9,), 7.0, dtype=dtype, device=DEV)
    out = torch.as_strided(whole, (5, 1000), (stride, 1), offset)
    got = atspeed_distill_grad(c["logits"], c["teacher_index"], atspeed_distill_loss(**c)[1], None, c["temperature"], out=out)
    assert got is out and torch.equal(out, grad)
    out.fill_(7.0)
    assert bool((whole == 7.0).all())


@pytest.mark.parametrize("tail,reverse", FORMS)
def test_a_student_that_is_sure_keeps_its_rest(tail, reverse):
    """Nearly all of q in the tops: the rest's share and 1 - p_rest / q_rest keep their digits."""
    c = case(3, 8, 2000, 5, F32, tail, reverse)
    top = c["teacher_index"].long().clamp(min=0)
    c["logits"].scatter_(1, top, 18.0 + torch.arange(5, device=DEV).expand(8, 5))
    check(c)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tail,reverse", FORMS)
def test_masked_columns(dtype, tail, reverse):
    """-infinity in the student's and the teacher's logits: no share, no top."""
    c = case(4, 7, 600, 8, dtype, tail, reverse)
    keep = torch.zeros((7, 600), dtype=torch.bool, device=DEV)
    keep.scatter_(1, c["teacher_index"].long().clamp(min=0), True)
    drop = (torch.rand((7, 600), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)) < 0.7) & ~keep
    c["logits"].masked_fill_(drop, -math.inf)
    c["teacher_logit"][1, 2:] = -math.inf
    c["teacher_index"][2, 1:] = -1
    _, grad = check(c)
    assert not bool(grad[drop].any())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_masked_top_costs_infinity_and_has_a_gradient(dtype):
    c = case(5, 3, 300, 6, dtype)
    c["logits"].scatter_(1, c["teacher_index"][:, 1:2].long().clamp(min=0), -math.inf)
    c["teacher_index"][:, 1].clamp_(min=0)
    loss, _ = check(c)
    assert bool((loss == math.inf).all())
    check(dict(c, reverse=True))                               # q is 0 there: nothing


def test_rows_of_nothing_but_minus_infinity():
    for tail, reverse in FORMS:
        c = case(6, 3, 300, 6, F32, tail, reverse)
        c["logits"][1] = -math.inf
        loss, grad = check(c)
        assert (float(loss[1]) == 0.0) if reverse else (float(loss[1]) == math.inf)
        assert bool(torch.isfinite(grad).all())


def test_no_rest_in_the_student():
    """Every column outside the tops is -infinity: the forward form is infinite with a tail, none has a NaN gradient."""
    for tail, reverse in FORMS:
        c = case(7, 3, 200, 6, F32, tail, reverse)
        inside = torch.zeros((3, 200), dtype=torch.bool, device=DEV)
        inside.scatter_(1, c["teacher_index"].long().clamp(min=0), True)
        c["logits"].masked_fill_(~inside, -math.inf)
        check(c)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tail,reverse", FORMS)
def test_rows_that_do_not_count_are_zero_whatever_they_hold(dtype, tail, reverse):
    c = case(8, 6, 5000, 7, dtype, tail, reverse)
    c["weight"][1] = 0.0
    c["teacher_index"][3] = torch.tensor([-1, 5000, 2 ** 31 - 1, -2 ** 31, -5, 5001, -1], device=DEV)
    c["teacher_logit"][4] = -math.inf
    for r in (1, 3, 4):
        c["logits"][r, ::7] = math.nan
        c["logits"][r, 1] = math.inf
    c["teacher_logit"][3] = math.nan
    loss, grad = check(c, torch.tensor([1.0, math.nan, 1, math.inf, 2, 1], device=DEV))
    assert not bool(loss[[1, 3, 4]].any()) and not bool(grad[[1, 3, 4]].any())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nan_in_a_row_stays_in_it(dtype):
    for tail, reverse in FORMS:
        c = case(9, 6, 3000, 7, dtype, tail, reverse)
        clean_loss, clean = check(c)
        x = dict(c, logits=c["logits"].clone())
        x["logits"][1, 2999] = math.nan
        x["logits"][2, 0] = math.inf
        x["logits"][4, 5], x["logits"][4, 2000] = math.nan, math.inf
        loss, saved = atspeed_distill_loss(**x)
        grad = atspeed_distill_grad(x["logits"], x["teacher_index"], saved)
        for r in range(6):
            if r in (1, 2, 4):
                assert math.isnan(float(loss[r])) and bool(torch.isnan(grad[r]).all())
            else:
                assert torch.equal(loss[r], clean_loss[r]) and torch.equal(grad[r], clean[r])


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("m", [7, 100])
def test_a_teacher_that_is_no_number_makes_its_row_nan(bad, m):
    for tail, reverse in FORMS:
        c = case(10, 5, 900, m, F32, tail, reverse)
        c["teacher_index"][1] = torch.arange(m, device=DEV) * 3
        clean_loss, clean = check(c)
        x = dict(c, teacher_logit=c["teacher_logit"].clone())
        x["teacher_logit"][1, m - 1] = bad
        rows = [1]
        if tail:
            x["tail"] = c["tail"].clone()
            x["tail"][3] = bad
            rows.append(3)
        loss, saved = atspeed_distill_loss(**x)
        grad = atspeed_distill_grad(x["logits"], x["teacher_index"], saved)
        for r in range(5):
            if r in rows:
                assert math.isnan(float(loss[r])) and bool(torch.isnan(grad[r]).all())
            else:
                assert torch.equal(loss[r], clean_loss[r]) and torch.equal(grad[r], clean[r])


def test_padded_teachers_may_hold_nan():
    c = case(10, 4, 400, 8)
    c["teacher_index"][:, 5:] = -1
    c["teacher_logit"][:, 5:] = math.nan
    check(c)


def test_every_index_the_same():
    c = case(11, 3, 100, 200)
    c["teacher_index"][:] = 17
    _, grad = check(c)
    assert bool((grad[:, 17] != 0).all())


@pytest.mark.parametrize("tail,reverse", FORMS)
def test_gradient_against_differences_of_the_loss(tail, reverse):
    """Along random directions of entries within 1; T = 1, weights 1.

    A divergence is a sum of log-sum-exps of q and of parts of it (forward: coefficients 1 and p_rest), whose third
    derivatives along a direction within 1 are at most 0.77 each (of a variable within 1, range 2): 1.54 h^2 / 6.  The
    reverse form's are bounded by the ones measured on the 64-bit definition at the same points.
    """
    c = case(12, 16, 500, 9, F32, tail, reverse, weight=False)
    grad = atspeed_distill_grad(c["logits"], c["teacher_index"], atspeed_distill_loss(**c)[1]).double()
    u = torch.rand((16, 500), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2)) * 2 - 1
    h = 2.0 ** -5
    sides, exact = [], []
    for sign in (1, -1):
        x = dict(c, logits=c["logits"] + sign * h * u)
        sides.append(atspeed_distill_loss(**x)[0].double())
        w, _, off, _ = ref.distill(num(x["logits"]), num(c["teacher_logit"]), num(c["teacher_index"]).astype(int),
                                   num(c["tail"]), None, 1.0, reverse)
        exact.append((w, off))
    slope = ((sides[0] - sides[1]) / (2 * h)).cpu().numpy()
    along = (grad * u.double()).sum(1).cpu().numpy()
    room = (exact[0][1] + exact[1][1]) / (2 * h) + 1e-5 * np.abs(grad.cpu().numpy()).sum(1)
    if reverse:
        room = room + np.abs((exact[0][0] - exact[1][0]) / (2 * h) - along)
    else:
        room = room + 1.54 * h * h / 6
    assert (np.abs(slope - along) <= room).all() and (room < 0.05 * (0.02 + np.abs(along).max())).all()


def test_autograd_of_a_draft():
    """Through a linear head in fp32: the gradients of the weights are those of the formula's logits."""
    g = torch.Generator(device=DEV).manual_seed(3)
    h = torch.randn((20, 32), generator=g, device=DEV)
    w = torch.randn((300, 32), generator=g, device=DEV, requires_grad=True)
    c = case(13, 20, 300, 8, T=2.0)
    c.pop("logits")
    logits = h @ w.t()
    loss = distill(logits, **c)
    up = torch.rand(20, device=DEV) + 0.5
    (loss * up).sum().backward()
    x = logits.detach()
    direct, saved = atspeed_distill_loss(x, **c)
    grad = atspeed_distill_grad(x, c["teacher_index"], saved, up, 2.0)
    assert torch.equal(loss.detach(), direct)
    torch.testing.assert_close(w.grad, grad.t() @ h, rtol=0, atol=0)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(torch.autograd.grad(distill(h @ w.t(), **c).sum(), w, create_graph=True)[0].sum(), w)
    # a loss that expands (every row the same upstream gradient, stride 0)
    w.grad = None
    distill(h @ w.t(), **c).sum().backward()
    ones = atspeed_distill_grad(x, c["teacher_index"], saved, None, 2.0)
    torch.testing.assert_close(w.grad, ones.t() @ h, rtol=0, atol=0)


def test_saved_logits_are_watched():
    c = case(14, 10, 200, 8)
    x = c.pop("logits").clone().requires_grad_()
    loss = distill(x, **c)
    with torch.no_grad():
        x.mul_(0.5)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()


def test_repeats_on_streams_and_in_graphs():
    """Loss and gradient, alternating on two streams and captured in two graphs, equal the eager calls."""
    cases = [case(15 + i, 30, 9000 + i, 20, BF16, True, bool(i)) for i in range(2)]

    def both(c):
        loss, saved = atspeed_distill_loss(**c)
        return loss, atspeed_distill_grad(c["logits"], c["teacher_index"], saved, None, c["temperature"])

    want = [both(c) for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(device=DEV) for _ in cases], []
    for _ in range(5):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                got.append((i, both(c)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i, g in got for a, b in zip(g, want[i]))
    graphs, outs = [torch.cuda.CUDAGraph() for _ in cases], []
    for g, c in zip(graphs, cases):
        with torch.cuda.graph(g):
            outs.append(both(c))
    for _ in range(3):
        for g, o, w in zip(graphs, outs, want):
            for t in o:
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(o, w))


def test_a_training_step_in_a_graph():
    """Forward, loss, backward and a step of a head captured after warm-up on a side stream; replays follow the eager one."""
    g = torch.Generator(device=DEV).manual_seed(4)
    h = torch.randn((24, 16), generator=g, device=DEV)
    c = case(17, 24, 150, 6)
    c.pop("logits")
    start = torch.randn((150, 16), generator=g, device=DEV)

    def step(w):
        grad, = torch.autograd.grad(distill(h @ w.t(), **c).sum(), w)
        with torch.no_grad():
            w -= 0.05 * grad
        return grad

    eager, graphed = start.clone().requires_grad_(), start.clone().requires_grad_()
    side = torch.cuda.Stream(device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step(graphed)
    torch.cuda.current_stream().wait_stream(side)
    with torch.no_grad():
        graphed.copy_(start)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(graphed)
    for _ in range(4):
        graph.replay()
        want = step(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(graphed, eager)


def test_rows_long_enough_to_need_more_lds_in_a_graph():
    c = case(21, 3, 600_000, 30, BF16)
    want = check(c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, saved = atspeed_distill_loss(**c)
        grad = atspeed_distill_grad(c["logits"], c["teacher_index"], saved)
    for _ in range(3):
        loss.zero_(), grad.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(grad, want[1])


@pytest.mark.parametrize("m", [1, 64, 65, 256])
@pytest.mark.parametrize("tail,reverse", FORMS)
@pytest.mark.parametrize("rows", [2, 1200])
def test_every_size_of_workgroup(m, tail, reverse, rows):
    """Few long rows, many of them, tops of one wave and of several."""
    c = case(22 + m, rows, 17000 if rows == 2 else 600, m, BF16, tail, reverse)
    c["teacher_index"][0] = torch.arange(m, device=DEV).int() // 2       # every column twice
    check(c)


def test_offsets_past_32_bits():
    stride = (1 << 31) + 8
    whole = torch.empty(2 * stride + 700, dtype=BF16, device=DEV)
    c = case(18, 3, 700, 9, BF16)
    far = torch.as_strided(whole, (3, 700), (stride, 1))
    far.copy_(c["logits"])
    want = check(c)
    loss, saved = atspeed_distill_loss(**dict(c, logits=far))
    out = torch.as_strided(torch.empty_like(whole), (3, 700), (stride, 1))
    atspeed_distill_grad(far, c["teacher_index"], saved, out=out)
    assert torch.equal(loss, want[0]) and torch.equal(out, want[1])


def test_many_columns():
    """2^20 columns: the most."""
    for dtype in (F32, BF16):
        check(case(19, 2, 1 << 20, 50, dtype))


def test_refusals():
    c = case(20, 4, 50, 3)
    good, saved = atspeed_distill_loss(**c)
    for kw in (dict(teacher_logit=c["teacher_logit"].bfloat16()), dict(teacher_logit=c["teacher_logit"][:, :2]),
               dict(teacher_index=c["teacher_index"].long()), dict(teacher_index=c["teacher_index"][0]),
               dict(tail=c["tail"][:2]), dict(weight=c["weight"].double()), dict(logits=c["logits"].half()),
               dict(logits=c["logits"][0]), dict(logits=c["logits"].t()), dict(weight=c["weight"].cpu())):
        with pytest.raises(ValueError):
            atspeed_distill_loss(**{**c, **kw})
    for kw in (dict(temperature=0.0), dict(temperature=math.nan), dict(reverse=True, tail=None),
               dict(teacher_index=c["teacher_index"][:, :0], teacher_logit=c["teacher_logit"][:, :0])):
        with pytest.raises(AtspeedError):
            atspeed_distill_loss(**{**c, **kw})
    x, i = c["logits"], c["teacher_index"]
    for call in (lambda: atspeed_distill_grad(x, i, saved[:, :4]), lambda: atspeed_distill_grad(x, i, saved, good[:2]),
                 lambda: atspeed_distill_grad(x, i, saved, out=x.bfloat16()),
                 lambda: atspeed_distill_grad(x, i, saved, out=x[:2])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(AtspeedError):
        atspeed_distill_grad(x, i, saved, out=x)

"""Distillation where the teacher's logits lie far apart, where the student's rest is next to
nothing, and where a row holds no numbers: against the definition in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2410_05165_amd.align import atspeed_distill_grad, atspeed_distill_loss  # noqa: E402
from test_gpu_distill import BF16, DEV, F32, FORMS, case, check  # noqa: E402


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tail,reverse", FORMS)
@pytest.mark.parametrize("m", [6, 100])
@pytest.mark.parametrize("T,far", [(1.0, 720.0), (1.0, 1000.0), (1.0, 1e4), (0.01, 15.0), (1.0, math.inf)])
def test_teacher_logits_far_below_the_best(dtype, tail, reverse, m, T, far):
    """Finitely masked teachers (infinity: the type's lowest number), columns named twice among them, a far tail."""
    c = case(31, 6, 700, m, dtype, tail, reverse, T, spread=1.0, weight=far < math.inf)   # 3.4e38 times 2 has no fp32
    c["logits"].mul_(T)
    c["teacher_logit"].mul_(T)
    low = torch.finfo(dtype).min if far == math.inf else -far
    c["teacher_logit"][0, 1] = low
    c["teacher_logit"][1, 2:] = low
    c["teacher_logit"][2, 0] = c["teacher_logit"][2, 3] = low      # one column
    c["teacher_index"][2, 3] = c["teacher_index"][2, 0]
    c["teacher_logit"][3] = low
    c["teacher_index"][4, 4] = c["teacher_index"][4, 1]
    c["teacher_logit"][4, 1] = low                                 # one column, far apart
    if tail:
        c["tail"] = torch.logsumexp(c["teacher_logit"].double() / T, 1).float() - 1.0
        c["tail"][5] = -far / T if far < math.inf else torch.finfo(F32).min
    check(c)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("gap", [60.0, 80.0, 86.0])
def test_gradients_of_scaled_losses_over_a_rest_of_next_to_nothing(dtype, reverse, gap):
    """A student that is sure of its tops, most other columns masked, the loss scaled up: no NaN, and the columns that
    are left keep their gradient."""
    c = case(32, 5, 900, 6, dtype, True, reverse, spread=1.0, weight=False)
    c["teacher_index"][:] = 7 * torch.arange(6, device=DEV) + 3
    inside = torch.zeros((5, 900), dtype=torch.bool, device=DEV)
    inside.scatter_(1, c["teacher_index"].long(), True)
    c["logits"].masked_fill_(~inside, -math.inf)
    left = torch.zeros_like(inside)
    left[:, 11::100] = True
    c["logits"][left] = c["logits"].masked_fill(~inside, -math.inf).amax(1)[:, None].expand(5, 900)[left] - gap
    c["logits"][:, 5::90] = torch.finfo(dtype).min             # masked by a number
    for scale in (1.0, 65536.0, 2.0 ** 100):
        _, grad = check(c, torch.full((5,), scale, device=DEV))
        assert bool(torch.isfinite(grad).all())
        assert bool((grad[left] != 0).all()) or reverse
        assert not bool(grad[~inside & ~left].any())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("tail,reverse", FORMS)
@pytest.mark.parametrize("m", [7, 100])
def test_a_teacher_that_is_no_number_beside_masked_students(bad, tail, reverse, m):
    """Where the student's rest, one of its tops or all of its logits are -infinity, the row is NaN as any other."""
    c = case(33, 5, 900, m, F32, tail, reverse)
    c["teacher_index"][:] = torch.arange(m, device=DEV) * 3
    c["teacher_index"][:, 1] = 0                               # twice
    inside = torch.zeros((5, 900), dtype=torch.bool, device=DEV)
    inside.scatter_(1, c["teacher_index"].long(), True)
    c["logits"][0] = torch.where(inside[0], c["logits"][0], -math.inf)
    c["logits"][1] = -math.inf
    c["logits"][2, 6] = -math.inf
    rows = [0, 1, 2]
    c["teacher_logit"][:3, m - 1] = bad
    loss, saved = atspeed_distill_loss(**c)
    grad = atspeed_distill_grad(c["logits"], c["teacher_index"], saved)
    for r in range(5):
        assert math.isnan(float(loss[r])) == (r in rows)
        assert bool(torch.isnan(grad[r]).all()) if r in rows else bool(torch.isfinite(grad[r]).all())
    if tail:
        c["teacher_logit"][:3, m - 1] = 0.0
        c["tail"][:3] = bad
        loss, saved = atspeed_distill_loss(**c)
        grad = atspeed_distill_grad(c["logits"], c["teacher_index"], saved)
        for r in rows:
            assert math.isnan(float(loss[r])) and bool(torch.isnan(grad[r]).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_student_logits_further_apart_than_fp32_reaches(dtype):
    """A top 5e38 below the largest logit: the forward form takes p times that distance, not infinity."""
    c = case(34, 4, 300, 5, dtype, False, False, weight=False)
    c["teacher_index"][:] = torch.arange(5, device=DEV) * 11 + 2
    c["teacher_logit"][:] = torch.tensor([2.0, 1.0, -6.0, -7.0, -5.0], device=DEV)
    c["logits"][1:, 2] = 2.5e38
    c["logits"][1, 24] = -2.5e38
    c["logits"][2:, 35] = -2.5e38
    loss, _ = check(c)
    assert bool(torch.isfinite(loss).all())

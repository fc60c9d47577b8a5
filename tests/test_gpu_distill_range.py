"""Distillation where logits lie far apart, against the definition in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

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

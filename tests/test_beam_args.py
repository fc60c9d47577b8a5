"""Beam selection, forked pages, moved tokens and distillation: their structures match the
header, and every argument error is found on the host before any launch (no GPU needed)."""
import ctypes as C

import pytest

from paper_2410_05165_amd import binding as bd
from test_paged_args import INVALID, OK, P, SHAPE, WORKSPACE, fill, refuse, test_structures_follow_the_header as follows


@pytest.mark.parametrize("cls,name", [(bd.BeamSelectArgs, "beam_select"), (bd.PageForkArgs, "page_fork"),
                                      (bd.PageCopyArgs, "page_copy"), (bd.KvCompactArgs, "kv_compact"),
                                      (bd.DistillLossArgs, "distill_loss"), (bd.DistillGradArgs, "distill_grad")])
def test_structures(cls, name):
    follows(cls, f"atspeed_{name}_args")


BEAM = dict(dtype=bd.BF16, B=3, n_rows=12, n_cols=500, k=10, n_paths=12, max_path=4, logits_stride=500)
FORK = dict(B=4, page_size=16, max_pages=8, n_pool=40)
CACHE = dict(n_layers=2, n_kv_heads=2, d_head=128, page_size=16, n_pool=10, dtype=bd.BF16, k_page=4096, k_token=256,
             k_head=128, v_page=4096, v_token=256, v_head=128, k_layer_stride=40960, v_layer_stride=40960)
LOSS = dict(dtype=bd.FP32, n_rows=5, n_cols=100, n_tops=8, temperature=1.0, logits_stride=100)
GRAD = dict(LOSS, grad_stride=100)
nulls = lambda *names: [(INVALID, {n: None}) for n in names]  # noqa: E731


def test_beam_refusals():
    bad = [(INVALID, dict(dtype=2)), (INVALID, dict(B=0)), (INVALID, dict(B=1025)), (INVALID, dict(n_rows=-1)),
           (INVALID, dict(n_cols=0)), (INVALID, dict(n_cols=2 ** 20 + 1)), (INVALID, dict(k=0)), (INVALID, dict(k=257)),
           (SHAPE, dict(logits_stride=499)), (INVALID, dict(n_paths=0)), (INVALID, dict(max_path=0)),
           (INVALID, dict(max_path=2 ** 16 + 1)), (INVALID, dict(score=P, score_out=P)),
           (INVALID, dict(paths=P, paths_out=P)), (INVALID, dict(path_len=P, path_len_out=P)),
           (SHAPE, dict(n_rows=2 ** 27))]
    bad += nulls("logits", "row_off", "count", "parent", "token", "score_out", "path_len", "paths", "paths_out",
                 "path_len_out")
    refuse("atspeed_beam_select", bd.BeamSelectArgs, BEAM, bad, P, 1 << 40)
    lib, n = bd.load_library(), C.c_size_t(0)
    size = lib.atspeed_beam_select_workspace_bytes
    assert size(C.byref(fill(bd.BeamSelectArgs, **BEAM)), C.byref(n)) == OK and n.value > 0
    assert size(C.byref(fill(bd.BeamSelectArgs, **BEAM)), None) == INVALID
    assert size(C.byref(fill(bd.BeamSelectArgs, **{**BEAM, "k": 0})), C.byref(n)) == INVALID
    for ws, room in ((None, n.value), (P + 8, n.value), (P, n.value - 1)):
        assert lib.atspeed_beam_select(C.byref(fill(bd.BeamSelectArgs, **BEAM)), ws, C.c_size_t(room), None) == WORKSPACE


def test_fork_refusals():
    bad = [(INVALID, dict(B=0)), (INVALID, dict(B=1025)), (INVALID, dict(page_size=0)), (INVALID, dict(page_size=24)),
           (INVALID, dict(page_size=2048)), (INVALID, dict(n_pool=0)), (SHAPE, dict(n_pool=2 ** 27)),
           (INVALID, dict(max_pages=0)), (SHAPE, dict(B=1024, max_pages=2 ** 21)), (INVALID, dict(held=P, length=P)),
           (INVALID, dict(src=P, copy_src=P)), (INVALID, dict(keep=P, block_table=P))]
    bad += nulls("held", "block_table", "free_pages", "n_free", "shared", "length", "refused", "copy_src", "copy_dst",
                 "copy_len")
    refuse("atspeed_page_fork", bd.PageForkArgs, FORK, bad, P, 1 << 40)
    lib, n = bd.load_library(), C.c_size_t(0)
    assert lib.atspeed_page_fork_workspace_bytes(C.byref(fill(bd.PageForkArgs, **FORK)), C.byref(n)) == OK
    for ws, room in ((None, n.value), (P + 4, n.value), (P, n.value - 1)):
        assert lib.atspeed_page_fork(C.byref(fill(bd.PageForkArgs, **FORK)), ws, C.c_size_t(room), None) == WORKSPACE


@pytest.mark.parametrize("call,cls,more,own", [
    ("atspeed_page_copy", bd.PageCopyArgs, dict(n=3), [(INVALID, dict(n=-1)), (SHAPE, dict(n=2 ** 23))]),
    ("atspeed_kv_compact", bd.KvCompactArgs, dict(B=3, max_pages=5, max_path=6),
     [(INVALID, dict(B=0)), (INVALID, dict(B=1025)), (INVALID, dict(max_pages=0)), (INVALID, dict(max_path=0)),
      (INVALID, dict(max_path=4097))])])
def test_move_refusals(call, cls, more, own):
    bad = own + [(INVALID, dict(dtype=2)), (SHAPE, dict(d_head=32)), (SHAPE, dict(d_head=96)), (INVALID, dict(n_kv_heads=0)),
                 (INVALID, dict(page_size=3)), (INVALID, dict(n_pool=0)), (INVALID, dict(n_layers=0)),
                 (INVALID, dict(n_layers=1025)), (INVALID, dict(k_page=4097)), (INVALID, dict(v_token=2)),
                 (INVALID, dict(k_head=4)), (INVALID, dict(k_layer_stride=3)), (INVALID, dict(v_layer_stride=12)),
                 (INVALID, dict(k_data=P + 8)), (INVALID, dict(v_data=P + 2))]
    bad += nulls("k_data", "v_data", *(("src", "dst", "length") if "n" in more else ("block_table", "ctx", "path", "n_path")))
    refuse(call, cls, {**CACHE, **more}, bad)
    if "n" in more:
        assert getattr(bd.load_library(), call)(C.byref(fill(cls, **{**CACHE, "n": 0})), None) == OK


def test_distill_refusals():
    both = [(INVALID, dict(dtype=2)), (INVALID, dict(n_rows=-1)), (INVALID, dict(n_cols=0)), (INVALID, dict(n_cols=2 ** 20 + 1)),
            (INVALID, dict(n_tops=0)), (INVALID, dict(n_tops=257)), (INVALID, dict(temperature=0.0)),
            (INVALID, dict(temperature=-1.0)), (INVALID, dict(temperature=float("nan"))),
            (INVALID, dict(temperature=float("inf"))), (INVALID, dict(temperature=1e-40)), (SHAPE, dict(logits_stride=99)), (SHAPE, dict(n_rows=2 ** 24))]
    refuse("atspeed_distill_loss", bd.DistillLossArgs, LOSS,
           both + [(INVALID, dict(reverse=1, tail=None))] + nulls("logits", "teacher_logit", "teacher_index", "loss", "saved"))
    refuse("atspeed_distill_grad", bd.DistillGradArgs, GRAD,
           both + [(SHAPE, dict(grad_stride=99)), (INVALID, dict(logits=P, grad=P))]
           + nulls("logits", "teacher_index", "saved", "grad"))
    lib = bd.load_library()
    assert lib.atspeed_distill_loss(C.byref(fill(bd.DistillLossArgs, **{**LOSS, "n_rows": 0})), None) == OK
    assert lib.atspeed_distill_grad(C.byref(fill(bd.DistillGradArgs, **{**GRAD, "n_rows": 0})), None) == OK


def test_tensors_that_are_not_on_a_gpu_are_refused():
    import torch
    from paper_2410_05165_amd import align, paged
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    x, c = torch.zeros(2, 5), torch.zeros(2, 3, 16, 1, 64)
    for call in (lambda: paged.atspeed_beam_select(x, i(2), 2),
                 lambda: paged.atspeed_page_fork(i(2), None, i(2, 3), i(5), i(1), i(5), 16),
                 lambda: paged.atspeed_page_copy(c, c, i(1), i(1), i(1)),
                 lambda: paged.atspeed_page_copy(c[0], c[0], i(1), i(1), i(1)),
                 lambda: paged.atspeed_kv_compact(c, c, i(2, 3), i(2), i(2, 4), i(2)),
                 lambda: align.atspeed_distill_loss(x, x, i(2, 5)),
                 lambda: align.atspeed_distill_grad(x, i(2, 5), torch.zeros(2, 7))):
        with pytest.raises(ValueError):
            call()


def test_distill_wants_a_teacher_without_gradient():
    import torch
    from paper_2410_05165_amd.align import distill
    i = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(ValueError, match="teacher_logit"):
        distill(torch.zeros(2, 5), torch.zeros(2, 3, requires_grad=True), i)
    with pytest.raises(ValueError, match="weight"):
        distill(torch.zeros(2, 5), torch.zeros(2, 3), i, weight=torch.ones(2, requires_grad=True))

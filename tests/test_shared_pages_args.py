"""What PagedKV.plan looks at before it forks (no GPU needed for tensors that are on none)."""
import pytest
import torch

from paper_2410_05165_amd import paged


def test_plans_of_caches_on_no_gpu_are_refused_before_the_fork():
    kv = paged.PagedKV(2, 6, 4, 1, 64, 2, 8, device="cpu", share=True)
    add = torch.zeros(2, dtype=torch.int32)
    for wrong in (dict(), dict(add=None), dict(max_rows=-1), dict(parent=add)):
        before = {n: getattr(kv, n).clone() for n in ("length", "block_table", "free_pages", "n_free", "shared")}
        with pytest.raises((ValueError, TypeError)):
            kv.plan(**{**dict(keep=None, add=add, max_rows=4), **wrong})
        for n, x in before.items():
            assert torch.equal(getattr(kv, n), x), n


def test_compact_keep_refusals():
    import ctypes as C
    from paper_2410_05165_amd import binding as bd
    from test_beam_args import CACHE
    from test_paged_args import INVALID, P, fill, refuse
    good = {**CACHE, "B": 3, "max_pages": 5, "max_path": 6}
    more = C.c_void_p(P), C.c_void_p(P + 4096)
    refuse("atspeed_kv_compact_keep", bd.KvCompactArgs, good,
           [(INVALID, dict(dtype=2)), (INVALID, dict(B=0)), (INVALID, dict(max_path=4097)), (INVALID, dict(ctx=None)),
            (INVALID, dict(ctx=P + 4096)), (INVALID, dict(n_path=P + 4096)), (INVALID, dict(path=P + 4096))], *more)
    call = bd.load_library().atspeed_kv_compact_keep
    for length, keep in ((None, P), (P, None), (P, P)):
        assert call(C.byref(fill(bd.KvCompactArgs, **good)), C.c_void_p(length), C.c_void_p(keep), None) == INVALID

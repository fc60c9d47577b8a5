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

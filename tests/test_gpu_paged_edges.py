"""Edges of the paged operators: malformed requests."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_paged import DEV, ints  # noqa: E402
from paper_2410_05165_amd.paged import atspeed_logit_rules, atspeed_page_plan  # noqa: E402


# ---------------------------------------------------------------- step plan

def overfull_plan(add):
    """Three requests of at most 6 nodes, the second with `add` rows."""
    new, parent = [4, add, 6], np.full((3, 6), -1)
    parent[:, 1:] = np.arange(5)
    p = atspeed_page_plan(ints([0, 8, 3]), ints([0, 8, 3]), ints(new), ints(np.arange(12).reshape(3, 4)),
                          ints(np.arange(12, 24)), ints([5]), 8, 40, ints(parent))
    return p, np.minimum(np.concatenate([[0], np.cumsum(new)]), 40)


@pytest.mark.parametrize("add", [7, 9, 13, 30])
def test_rows_past_a_requests_nodes_have_no_tree_slot(add):
    """A request with more rows than nodes is refused; its rows past them are no rows of the padded array."""
    p, off = overfull_plan(add)
    assert p.refused.cpu().tolist() == [0, 2, 0]
    want = [b * 6 + i if i < 6 else -1 for b in range(3) for i in range(off[b + 1] - off[b])]
    assert p.tree_slot.cpu().tolist() == want + [-1] * (40 - len(want))


@pytest.mark.parametrize("add", [7, 9, 13, 30])
def test_a_malformed_request_leaves_its_neighbours_rows(add):
    """Logits scattered by the plan's tree slots: every other request finds its own in its own rows."""
    p, off = overfull_plan(add)
    g = torch.Generator(device=DEV).manual_seed(add)
    logits, out = torch.randn((40, 33), generator=g, device=DEV), torch.full((3, 6, 33), 7.0, device=DEV)
    atspeed_logit_rules(logits, p.row_off, out=out, out_row=p.tree_slot)
    for b in range(3):
        n = min(6, off[b + 1] - off[b])
        assert torch.equal(out[b, :n], logits[off[b]:off[b] + n]) and bool((out[b, n:] == 7.0).all()), b

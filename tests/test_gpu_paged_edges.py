"""Edges of the paged operators: malformed requests, rows whose only key is not finite, keys that are
not there, keys of other branches, and what probabilities keep of their 32 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import _paged_reference as ref  # noqa: E402
from test_gpu_paged import BF16, DEV, F32, TYPES, attention_case, ints  # noqa: E402
from paper_2410_05165_amd.paged import (PagedKV, atspeed_kv_append, atspeed_logit_rules,  # noqa: E402
                                        atspeed_page_plan, atspeed_tree_attention)


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


# ---------------------------------------------------------------- attention

def roots(c, n):
    """Every new row sees the context and itself alone."""
    rows = torch.arange(n, device=DEV)
    c["mask"] = torch.zeros((n, -(-n // 64)), dtype=torch.int64, device=DEV)
    c["mask"][rows, rows // 64] = torch.ones((), dtype=torch.int64, device=DEV) << (rows % 64)
    return c


def key_row(c, b, p):
    """Where key p of request b lies: page, token."""
    page = c["k_cache"].shape[1]
    return int(c["block_table"][b, p // page]), p % page


@pytest.mark.parametrize("dtype,dh", TYPES)
@pytest.mark.parametrize("ctx", [0, 5])
@pytest.mark.parametrize("n", [5, 40, 90, 150])
def test_a_row_whose_own_value_is_infinite(dtype, dh, ctx, n):
    """Rows that see their own key (and a few of the context) get the infinity of its value, whichever wave it falls to."""
    c = roots(attention_case(n + ctx, [ctx], [n], 4, 2, dh, 16, dtype, True), n)
    clean = atspeed_tree_attention(**c)
    for r in range(0, n, max(1, n // 12)):
        page, token = key_row(c, 0, ctx + r)
        kept = c["v_cache"][page, token, 0, 5].clone()
        for poison in (math.inf, -math.inf):
            c["v_cache"][page, token, 0, 5] = poison
            got = atspeed_tree_attention(**c)
            assert bool((got[r, :2, 5] == poison).all()), (r, got[r, :2, 5])
            got[r, :2, 5] = clean[r, :2, 5]
            assert torch.equal(got, clean)
        c["v_cache"][page, token, 0, 5] = kept


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (F32, 64)])
@pytest.mark.parametrize("n", [20, 70])
def test_infinite_values_in_pieces_that_begin_among_the_new_keys(dtype, dh, n):
    for ctx in range(4970, 5070, 17):
        c = roots(attention_case(ctx, [ctx, 9], [n, 0], 4, 2, dh, 16, dtype, True), n)
        clean = atspeed_tree_attention(**c)
        at = list(range(1, n, 6))
        for r in at:
            page, token = key_row(c, 0, ctx + r)
            c["v_cache"][page, token, 1, 3] = math.inf
        got = atspeed_tree_attention(**c)
        assert bool((got[at, 2:, 3] == math.inf).all()), ctx
        got[at, 2:, 3] = clean[at, 2:, 3]
        assert torch.equal(got, clean), ctx


def time_of(call):
    for _ in range(3):
        call()
    took = []
    for _ in range(9):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        took.append(a.elapsed_time(b))
    return sorted(took)[4]


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (F32, 64)])
@pytest.mark.parametrize("B,ctx,n", [(700, 690, 1), (100, 500, 70)])
def test_values_of_pages_that_are_not_a_requests_own_cost_it_nothing(dtype, dh, B, ctx, n):
    """Page 0 belongs to nobody and holds NaN: same bits, and no search through the requests' keys for them."""
    c = attention_case(7, [ctx + b % 60 for b in range(B)], [n] * B, 4, 2, dh, 16, dtype, n > 1)
    for name in ("k_cache", "v_cache"):
        c[name] = torch.cat([torch.zeros_like(c[name][:1]), c[name]])
    c["block_table"] = torch.where(c["block_table"] >= 0, c["block_table"] + 1, -1).int()
    clean, before = atspeed_tree_attention(**c), time_of(lambda: atspeed_tree_attention(**c))
    c["k_cache"][0], c["v_cache"][0] = math.nan, math.nan
    assert torch.equal(atspeed_tree_attention(**c), clean)
    after = time_of(lambda: atspeed_tree_attention(**c))
    # the same bits by the same instructions; a search of every key made it 12 to 22 times as long
    assert after < 2.5 * before, f"{before * 1e3:.1f} us with page 0 clean, {after * 1e3:.1f} with NaN in it"


@pytest.mark.parametrize("dtype,dh", TYPES)
@pytest.mark.parametrize("ctx,n", [(0, 30), (40, 3), (100, 60), (100, 150), (5000, 12), (5000, 70)])
def test_finite_keys_of_other_branches_do_not_move_a_row(dtype, dh, ctx, n):
    """A key that only its own row sees, however large, changes no bit of the others."""
    c = roots(attention_case(ctx + n, [ctx, 3], [n, 2], 4, 2, dh, 16, dtype, True, scale_q=4.0), n + 2)
    c["mask"][n:, 0] = torch.tensor([1, 3], device=DEV)
    clean, clean_lse = atspeed_tree_attention(**c, return_lse=True)
    for r in (0, n // 2, n - 1):
        page, token = key_row(c, 0, ctx + r)
        kept = c["k_cache"][page, token].clone()
        # along the row's own query: its score, and by chance others', rise by hundreds
        c["k_cache"][page, token] = (c["q"][r].view(2, 2, dh).sum(1).float() * 40).to(dtype)
        got, lse = atspeed_tree_attention(**c, return_lse=True)
        rest = [i for i in range(n + 2) if i != r]
        assert torch.equal(got[rest], clean[rest]) and torch.equal(lse[rest], clean_lse[rest]), r
        c["k_cache"][page, token] = kept


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("ctx,new,tree", [([50, 200], [1, 9], True), ([0, 300], [33, 20], True), ([300, 90], [257, 200], True),
                                          ([200, 10], [300, 150], False), ([9000, 700], [1, 1], False), ([7000, 300], [40, 60], True)])
def test_probabilities_keep_their_bits(dh, ctx, new, tree):
    """bf16: probabilities meet the values as their upper 16 bits, which leave less than 2^-7 of them, and what is
    left, rounded by at most 2^-8 of it: off by 2^-15.  The rest as in fp32 (scores, exponentials and sums: the
    bound of test_gpu_paged.close_to_exact), the output rounded once, 2^-8."""
    c = attention_case(sum(ctx) + sum(new), ctx, new, 8, 2, dh, 16, BF16, tree)
    got, lse = atspeed_tree_attention(**c, return_lse=True)
    out, want_lse, spread, reach = ref.attention(c["q"], c["k_cache"], c["v_cache"], c["block_table"], c["row_off"],
                                                 c["ctx"], c["mask"])
    e = (dh + 3) * 2.0 ** -24 * reach + 2.0 ** -21 * reach + 2.0 ** -22 + (c["max_ctx"] + c["max_new"] + 8) * 2.0 ** -24
    tol = 2.0 ** -8 * out.abs() + (2.0 ** -15 + 3 * e)[..., None] * spread
    off = (got.cpu().double() - out).abs()
    assert bool((off <= tol).all()), f"{int((off > tol).sum())} of {off.numel()}, worst {float((off / tol).max()):.2f} of the tolerance"


# ---------------------------------------------------------------- what autograd is told

def test_writes_are_seen_by_a_backward_pass_that_saved_the_tensor():
    """Each buffer that a call writes is saved by a product first: its backward pass refuses the new values."""
    c = attention_case(3, [20], [4], 4, 2, 64, 16, F32, True)
    table, free = c["block_table"], ints(np.arange(20))
    logits, off = torch.randn((4, 50), device=DEV), ints([0, 4])
    k = torch.randn((4, 2, 64), device=DEV)
    calls = [("k_cache", c["k_cache"], lambda: atspeed_kv_append(k, k, c["k_cache"], c["v_cache"], ints([0, 1, 2, 3]))),
             ("v_cache", c["v_cache"], lambda: atspeed_kv_append(k, k, c["k_cache"], c["v_cache"], ints([0, 1, 2, 3]))),
             ("a layer's caches", c["k_cache"], lambda: atspeed_kv_append(k, k, c["k_cache"][:], c["v_cache"][:], ints([0, 1, 2, 3]))),
             ("q in place", c["q"], lambda: atspeed_tree_attention(**c, out=c["q"])),
             ("logits in place", logits, lambda: atspeed_logit_rules(logits, off, out=logits))]
    for name, t, call in calls:
        x = torch.ones_like(t, requires_grad=True)
        loss = (x * t).sum()
        call()
        with pytest.raises(RuntimeError, match="inplace operation"):
            loss.backward()
    before = [t._version for t in (table, free)]
    atspeed_page_plan(ints([20]), ints([20]), ints([4]), table, free, ints([9]), 16, 4)
    assert all(t._version > v for t, v in zip((table, free), before))
    untouched = torch.randn((4, 50), device=DEV)
    x = torch.ones_like(untouched, requires_grad=True)
    loss = (x * untouched).sum()
    atspeed_logit_rules(untouched, off)
    loss.backward()                                      # read only
    with torch.inference_mode():
        caches = [torch.zeros((3, 16, 2, 64), device=DEV) for _ in range(2)]
    atspeed_kv_append(k, k, *caches, ints([0, 1, 2, 3]))   # tensors without versions
    assert torch.equal(caches[0].view(-1, 2, 64)[:4], k)


# ---------------------------------------------------------------- caches in captured steps

def test_captured_steps_of_a_cache_go_on_from_each_other():
    """PagedKV.plan, append and attention in a graph: replays and eager steps in turn equal eager steps alone."""
    rng = np.random.default_rng(5)
    g = torch.Generator(device=DEV).manual_seed(5)
    B, width, heads, kv, dh, page, pool = 5, 12, 4, 2, 64, 8, 60
    caches = [PagedKV(1, pool, page, kv, dh, B, 96, dtype=F32) for _ in range(2)]

    def inputs():
        r = lambda n: torch.randn((B * width, n, dh), generator=g, device=DEV)  # noqa: E731
        return dict(drop=ints(rng.integers(0, 5, B)), add=ints(rng.integers(0, width + 1, B)), q=r(heads), k=r(kv), v=r(kv))

    def step(cache, x):
        keep = torch.where(cache.length > 60, 0, (cache.length - x["drop"]).clamp(min=0)).int()
        p = cache.plan(keep, x["add"], B * width)
        cache.append(0, p, x["k"], x["v"])
        return p, cache.attention(0, p, x["q"], width, out=torch.zeros_like(x["q"]))

    hold = inputs()
    side = torch.cuda.Stream(device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(PagedKV(1, pool, page, kv, dh, B, 96, dtype=F32), hold)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(caches[0], hold)
    for i in range(12):
        x = inputs()
        want = step(caches[1], x)
        if i % 4 == 3:
            now = step(caches[0], x)                     # an eager step between the replays
        else:
            for k in hold:
                hold[k].copy_(x[k])
            graph.replay()
            now = got
        torch.cuda.synchronize()
        for a, b in zip(now[0][:-1], want[0][:-1]):
            assert torch.equal(a, b), i
        n = int(want[0].row_off[-1])
        assert torch.equal(now[1][:n], want[1][:n]), i
        for name in ("length", "n_free", "block_table", "k", "v"):
            assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), (i, name)
    held, t, free = (getattr(caches[0], n).cpu().numpy() for n in ("length", "block_table", "free_pages"))
    mine = [x for b in range(B) for x in t[b, :-(-held[b] // page)]]
    assert sorted(mine + list(free[:int(caches[0].n_free)])) == list(range(pool))


@pytest.mark.parametrize("made,used", [(True, False), (False, True), (True, True)])
def test_caches_in_and_out_of_inference_mode(made, used):
    with torch.inference_mode(made):
        cache = PagedKV(1, 20, 8, 2, 64, 2, 40, dtype=F32)
    k = torch.ones((7, 2, 64), device=DEV)
    with torch.inference_mode(used):
        for held in (0, 4, 9):
            p = cache.plan(ints([held, 0]), ints([5, 2]), 7)
            cache.append(0, p, k, k)
            out = cache.attention(0, p, torch.ones((7, 4, 64), device=DEV), 5)
            assert cache.length.tolist() == [held + 5, 2] and torch.equal(cache.length, p.length)
            assert bool((out == 1).all())

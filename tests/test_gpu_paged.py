"""The paged operators (step plan, cache append, tree attention, logit rules) against
plain implementations in Python integers and 64 bits."""
import math
import sys
import threading

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import _paged_reference as ref  # noqa: E402
from paper_2410_05165_amd.paged import (PagedKV, atspeed_kv_append, atspeed_logit_rules,  # noqa: E402
                                        atspeed_page_plan, atspeed_tree_attention)

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


# ---------------------------------------------------------------- step plan

def plan_case(rng, B, page, most, width, tree=True, bad=False):
    """Consistent page tables with requests that grow, shrink, end, start and (bad) are malformed."""
    held = rng.integers(0, most * page + 1, B)
    if B > 2:
        held[rng.integers(0, B)] = 0
        held[rng.integers(0, B)] = most * page
    before = -(-held // page)
    pool = int(before.sum()) + int(rng.integers(0, max(2, B * most // 4)))
    pool = max(pool, 1)
    order = rng.permutation(pool)
    table = np.full((B, most), -1, np.int64)
    at = 0
    for b in range(B):
        table[b, :before[b]] = order[at:at + before[b]]
        at += before[b]
    free = np.full(pool, -1, np.int64)
    free[:pool - at] = order[at:]
    keep = np.where(rng.random(B) < 0.5, held, rng.integers(0, held + 1))
    add = np.minimum(rng.integers(0, width + 1, B), np.maximum(0, most * page - keep))
    add[rng.random(B) < 0.2] = 0
    parent = np.stack([ref.tree_parents(rng, int(n), int(rng.integers(1, 7)), width) for n in add]) if tree else None
    if bad:
        for b in range(B):
            what = rng.integers(0, 12)
            if what == 0:
                keep[b] = held[b] + 1
            elif what == 1:
                add[b] = -3
            elif what == 2:
                held[b] = -1
            elif what == 3:
                add[b] = 2 ** 31 - 1
            elif what == 4 and tree and add[b] > 2:
                parent[b, 1] = 2                      # an ancestor that comes later
            elif what == 5 and tree and add[b] > 2:
                parent[b, add[b] - 1] = -7
            elif what == 6:
                held[b] = most * page + 1
    return held, keep, add, table, free, pool - at, parent


def check_plan(case, page, max_rows):
    held, keep, add, table, free, n_free, parent = case
    t, f = ints(table), ints(free)
    p = atspeed_page_plan(ints(held), ints(keep), ints(add), t, f, ints([n_free]), page, max_rows,
                          None if parent is None else ints(parent))
    want = ref.plan(held, keep, add, table, free, n_free, page, max_rows, parent)
    got = dict(table=t, n_free=p.n_free[0], length=p.length, ctx=p.ctx, refused=p.refused, row_off=p.row_off,
               row_user=p.row_user, row_pos=p.row_pos, slot=p.slot, tree_slot=p.tree_slot)
    for name, x in got.items():
        np.testing.assert_array_equal(x.cpu().numpy(), np.array(want[name]), err_msg=name)
    n = want["n_free"]
    np.testing.assert_array_equal(f.cpu().numpy()[:n], np.array(want["free"][:n], np.int64))
    if parent is not None:
        np.testing.assert_array_equal(p.mask.cpu().numpy(), want["mask"])
    return want


@pytest.mark.parametrize("B,page,most,width", [(1, 16, 1, 1), (1, 1, 40, 30), (3, 8, 5, 64), (7, 32, 4, 65),
                                               (64, 16, 9, 110), (255, 4, 6, 12), (257, 64, 3, 200), (1024, 16, 8, 40)])
@pytest.mark.parametrize("tree", [True, False])
def test_plan_equals_the_sequential_one(B, page, most, width, tree):
    rng = np.random.default_rng(B * 100 + page)
    for trial in range(2):
        case = plan_case(rng, B, page, most, width, tree)
        check_plan(case, page, max(0, int(case[2].sum())) + 5 * trial)


@pytest.mark.parametrize("seed", range(6))
def test_plan_with_malformed_requests_and_too_few_rows_or_pages(seed):
    rng = np.random.default_rng(seed)
    case = list(plan_case(rng, 40, 8, 6, 33, True, bad=True))
    if seed % 2:
        case[5] = min(case[5], 3)                      # hardly any free pages
    rows = int(np.maximum(np.minimum(case[2], 10 ** 6), 0).sum())
    want = check_plan(case, 8, rows // 2 if seed % 3 == 0 and rows < 10 ** 6 else 900)
    assert 2 in want["refused"]


@pytest.mark.parametrize("seed", range(4))
def test_plan_with_too_few_pages_refuses_the_later_requests(seed):
    rng = np.random.default_rng(seed)
    case = list(plan_case(rng, 40, 8, 6, 33, True))
    case[5] = min(case[5], 3)
    want = check_plan(case, 8, int(case[2].sum()))
    assert 1 in want["refused"] and 0 in want["refused"] and 2 not in want["refused"]


def test_plan_deep_paths_and_wide_masks():
    rng = np.random.default_rng(5)
    for width, n in ((1, 1), (64, 64), (300, 299), (1000, 1000)):
        parent = np.stack([np.arange(-1, width - 1), ref.tree_parents(rng, n, 9, width)]).astype(np.int32)
        case = (np.zeros(2, int), np.zeros(2, int), np.array([width, n]), np.full((2, 16), -1), np.arange(32), 32, parent)
        check_plan(case, 64, width + n)


def test_plan_survives_nonsense_state():
    """Table entries, the free list and its length hold garbage: every index stays inside."""
    rng = np.random.default_rng(9)
    B, most, page, pool = 50, 7, 8, 60
    held = rng.integers(0, most * page + 1, B)
    junk = lambda *s: ints(rng.integers(-2 ** 31, 2 ** 31, s))  # noqa: E731
    for n_free in (-5, 2 ** 31 - 1, 60):
        p = atspeed_page_plan(ints(held), ints(rng.integers(0, held + 1)), ints(rng.integers(0, 20, B)), junk(B, most),
                              junk(pool), ints([n_free]), page, 600, junk(B, 20))
        slot = p.slot.cpu().numpy()
        assert ((slot >= -1) & (slot < pool * page)).all()
        assert 0 <= int(p.n_free) <= pool


def test_plan_steps_keep_every_page_once():
    """Many steps: the pages of the tables and the free list are a permutation of the pool throughout."""
    rng = np.random.default_rng(3)
    B, page, pool = 20, 8, 90
    cache = PagedKV(1, pool, page, 1, 64, B, 100, dtype=F32)
    for step in range(25):
        held = cache.length.cpu().numpy()
        keep = np.where(rng.random(B) < 0.15, 0, np.maximum(0, held - rng.integers(0, 12, B)))
        add = np.minimum(rng.integers(0, 24, B), 100 - keep)
        p = cache.plan(ints(keep), ints(add), int(add.sum()))
        held, t, n = cache.length.cpu().numpy(), cache.block_table.cpu().numpy(), int(cache.n_free)
        mine = [x for b in range(B) for x in t[b, :-(-held[b] // page)]]
        assert sorted(mine + list(cache.free_pages.cpu().numpy()[:n])) == list(range(pool)), step
        refused = p.refused.cpu().numpy()
        assert (held == np.where(refused == 0, keep + add, held)).all()


# ---------------------------------------------------------------- append

@pytest.mark.parametrize("dtype,dh", [(BF16, 64), (BF16, 128), (F32, 32), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("heads,page,rows", [(1, 1, 1), (2, 16, 37), (12, 8, 100), (32, 64, 65)])
def test_append_writes_its_slots_only(dtype, dh, heads, page, rows):
    g = torch.Generator(device=DEV).manual_seed(rows)
    pool = rows // page + 3
    qkv = torch.randn((rows, 3 * heads * dh), generator=g, device=DEV).to(dtype)
    k, v = (qkv[:, i * heads * dh:(i + 1) * heads * dh].view(rows, heads, dh) for i in (1, 2))
    # one cache token-major, the other head-major
    kc = torch.randn((pool, page, heads, dh), generator=g, device=DEV).to(dtype)
    vc = torch.randn((pool, heads, page, dh), generator=g, device=DEV).to(dtype).transpose(1, 2)
    slot = torch.randperm(pool * page, generator=g, device=DEV)[:rows].int()
    slot[torch.rand(rows, generator=g, device=DEV) < 0.2] = -1
    if rows > 2:
        slot[1], slot[2] = pool * page, -2 ** 31
    want_k, want_v = kc.clone(), vc.clone()
    for r, s in enumerate(slot.tolist()):
        if 0 <= s < pool * page:
            want_k[s // page, s % page], want_v[s // page, s % page] = k[r], v[r]
    atspeed_kv_append(k, v, kc, vc, slot)
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


def test_append_beyond_32_bit_offsets():
    pool, page, heads, dh = 4200, 128, 32, 128            # 4.4 GB a cache, 2.2e9 elements
    kc = torch.zeros((pool, page, heads, dh), dtype=BF16, device=DEV)
    vc = torch.zeros((pool, page, heads, dh), dtype=BF16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn((5, heads, dh), generator=g, device=DEV).to(BF16) for _ in range(2))
    slot = ints([pool * page - 1, 0, 2 ** 31 // (heads * dh), 2 ** 31 // (heads * dh) - 1, 7])
    atspeed_kv_append(k, v, kc, vc, slot)
    at = slot.long()
    assert torch.equal(kc.view(-1, heads, dh)[at], k) and torch.equal(vc.view(-1, heads, dh)[at], v)
    assert int(kc.count_nonzero()) == int(k.count_nonzero())
    # and read back there by the attention: one row whose context sits in the last page
    table, off, ctx = ints([[pool - 1]]), ints([0, 1]), ints([page - 1])
    q = torch.randn((1, heads, dh), generator=g, device=DEV).to(BF16)
    kc[pool - 1], vc[pool - 1] = (torch.randn((page, heads, dh), generator=g, device=DEV).to(BF16) for _ in range(2))
    small = [c[pool - 1:].clone() for c in (kc, vc)]
    got = atspeed_tree_attention(q, kc, vc, table, off, ctx, page, 1)
    want = atspeed_tree_attention(q, *small, ints([[0]]), off, ctx, page, 1)
    assert torch.equal(got, want)


# ---------------------------------------------------------------- attention

def attention_case(seed, ctx, new, heads, kv_heads, dh, page, dtype, tree=True, levels=3, spare=0, scale_q=2.0):
    """Random caches behind shuffled pages, rows of each request, masks of random trees."""
    rng = np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    ctx, new = np.array(ctx), np.array(new)
    need = np.maximum(1, -(-(np.maximum(ctx, 0) + new) // page))
    most, pool = int(need.max()) + 1, int(need.sum()) + 3
    order = rng.permutation(pool)
    table = np.full((len(ctx), most), -1, np.int64)
    at = 0
    for b in range(len(ctx)):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    n = int(new.sum())
    rand = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)  # noqa: E731
    mask = None
    if tree:
        width = max(1, int(new.max()))
        parents = np.stack([ref.tree_parents(rng, int(m), levels, width) for m in new])
        mask = mask_of(parents, new, spare)
    q = (rand(n + spare, heads, dh).float() * scale_q).to(dtype)
    return dict(q=q, k_cache=rand(pool, page, kv_heads, dh), v_cache=rand(pool, page, kv_heads, dh),
                block_table=ints(table), row_off=ints(np.concatenate([[0], np.cumsum(new)])), ctx=ints(ctx),
                max_ctx=int(max(0, ctx.max())), max_new=int(new.max()), mask=mask)


def mask_of(parents, new, spare=0):
    width = parents.shape[1]
    out = np.zeros((int(new.sum()) + spare, -(-width // 64)), np.uint64)
    r = 0
    for b, n in enumerate(new):
        for i in range(n):
            j = i
            while j >= 0:
                out[r, j // 64] |= np.uint64(1) << np.uint64(j % 64)
                j = parents[b, j]
            r += 1
    return torch.from_numpy(out.view(np.int64)).to(DEV)


def close_to_exact(c, got, lse, scale=None):
    """Holds out and lse to the rounding of their computation.

    A score is a sum of d_head products and a scaling in fp32: off by at most e = (d_head + 3) 2^-24 sum|q k|
    scale, plus the rounding of the score for the exponential and of the exponential itself (together below
    2^-21 of the score's size and 2^-22).  Each probability is then off by the factor 1 + 2 e' with e' the
    sum of these, sums over n keys by n 2^-24, and in bf16 a probability is rounded by at most 2^-8.  What
    multiplies these is spread = sum p |v|.  The output is rounded once more, by 2^-8 (bf16) or 2^-24.
    """
    out, want_lse, spread, reach = ref.attention(c["q"], c["k_cache"], c["v_cache"], c["block_table"], c["row_off"],
                                                 c["ctx"], c["mask"], scale)
    dh, half = c["q"].shape[2], 2.0 ** -8 if c["q"].dtype is BF16 else 2.0 ** -24
    n_keys = c["max_ctx"] + c["max_new"]
    e = (dh + 3) * 2.0 ** -24 * reach + 2.0 ** -21 * reach + 2.0 ** -22 + (n_keys + 8) * 2.0 ** -24
    tol = half * out.abs() + ((half if half > 1e-4 else 0.0) + 3 * e)[..., None] * spread + 1e-30
    err = (got.cpu().double() - out).abs()
    live = int(c["row_off"][-1])
    assert bool((err[:live] <= tol[:live]).all()), f"worst {float((err / tol)[:live].max()):.2f} of its tolerance"
    if lse is not None:
        empty = want_lse[:live] == -math.inf
        got_lse = lse.cpu().double()[:live]
        assert bool((got_lse[empty] == -math.inf).all())
        off = (got_lse - want_lse[:live]).abs()[~empty]
        room = (e[:live] + 2.0 ** -22 * want_lse[:live].abs())[~empty]
        assert bool((off <= room).all()), f"lse: worst {float((off / room).max()):.2f}"


TYPES = [(BF16, 64), (BF16, 128), (F32, 32), (F32, 64), (F32, 128)]


@pytest.mark.parametrize("dtype,dh", TYPES)
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 4), (8, 2), (6, 2), (5, 1), (16, 1), (24, 1), (40, 2)])
@pytest.mark.parametrize("tree", [True, False])
def test_attention_head_layouts(dtype, dh, heads, kv_heads, tree):
    c = attention_case(heads * 7 + kv_heads, [37, 0, 129, 64], [20, 33, 1, 5], heads, kv_heads, dh, 16, dtype, tree)
    close_to_exact(c, *atspeed_tree_attention(**c, return_lse=True))


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (BF16, 64), (F32, 64)])
@pytest.mark.parametrize("page", [1, 8, 32, 64, 256, 1024])
@pytest.mark.parametrize("tree", [True, False])
def test_attention_pages(dtype, dh, page, tree):
    """Pages smaller than, equal to and larger than any tile; contexts that end everywhere in them."""
    c = attention_case(page, [0, 1, 63, 64, 65, 300], [3, 70, 1, 64, 65, 130], 4, 2, dh, page, dtype, tree)
    close_to_exact(c, *atspeed_tree_attention(**c, return_lse=True))


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (BF16, 64), (F32, 32)])
@pytest.mark.parametrize("new", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200, 257])
def test_attention_row_counts(dtype, dh, new):
    c = attention_case(new, [50, 200], [new, max(1, new - 1)], 2, 1, dh, 32, dtype, True, levels=4)
    close_to_exact(c, *atspeed_tree_attention(**c, return_lse=True))


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (BF16, 64), (F32, 64)])
@pytest.mark.parametrize("ctx", [511, 2000, 5003, 20000])
@pytest.mark.parametrize("new,tree", [(1, False), (9, True), (40, True)])
def test_attention_long_contexts(dtype, dh, ctx, new, tree):
    c = attention_case(ctx + new, [ctx, 3, ctx // 3], [new, new, 1], 8, 2, dh, 16, dtype, tree)
    close_to_exact(c, *atspeed_tree_attention(**c, return_lse=True))


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (F32, 64)])
def test_attention_of_an_empty_context_and_empty_rows(dtype, dh):
    """Requests without rows, without context, refused ones (-1), and rows whose mask is empty."""
    c = attention_case(4, [0, 12, -1, 0, 40], [6, 0, 9, 4, 7], 6, 3, dh, 8, dtype, True)
    c["mask"][2] = 0                      # no context and an empty mask: sees nothing
    c["mask"][15:19, :] = 0               # a whole request that sees nothing
    out, lse = atspeed_tree_attention(**c, return_lse=True)
    close_to_exact(c, out, lse)
    gone = [2] + list(range(6, 15)) + list(range(15, 19))
    assert bool((out[gone] == 0).all()) and bool((lse[gone] == -math.inf).all())


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (BF16, 64), (F32, 32), (F32, 128)])
@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
def test_attention_keeps_what_is_masked_out(dtype, dh, tree, poison):
    """NaN and infinities in the unread tail of pages, in unused pages and in rows that others do not see."""
    c = attention_case(11, [21, 70, 0], [30, 45, 17], 4, 2, dh, 16, dtype, tree, levels=2)
    page, table = 16, c["block_table"].cpu().numpy()
    off, ctx = c["row_off"].cpu().numpy(), c["ctx"].cpu().numpy()
    clean = atspeed_tree_attention(**c)
    held = torch.ones(c["k_cache"].shape[0] * page, dtype=torch.bool)
    for b in range(3):
        p = np.arange(ctx[b] + off[b + 1] - off[b])
        held[table[b, p // page] * page + p % page] = False
    hurt = []
    for cache in (c["k_cache"], c["v_cache"]):
        cache.view(-1, *cache.shape[2:])[held.to(DEV)] = poison
    assert torch.equal(atspeed_tree_attention(**c), clean)
    # the last row of each request: seen by itself alone, in a tree a leaf
    for b in range(3):
        r = int(off[b + 1]) - 1
        p = int(ctx[b] + r - off[b])
        slot = table[b, p // page] * page + p % page
        c["v_cache"].view(-1, *c["v_cache"].shape[2:])[slot] = poison
        c["k_cache"].view(-1, *c["k_cache"].shape[2:])[slot] = math.nan
        hurt.append(r)
    got = atspeed_tree_attention(**c)
    rest = [r for r in range(int(off[-1])) if r not in hurt]
    assert torch.equal(got[rest], clean[rest])
    assert bool(got[hurt].isnan().all())


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (BF16, 64), (F32, 32), (F32, 128)])
@pytest.mark.parametrize("new", [3, 40, 150])
@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
def test_attention_values_of_the_context_reach_every_row(dtype, dh, new, poison):
    """A value that is not finite in the context, in a tile with new keys or with a bad page too: every row has it."""
    c = attention_case(13, [100, 37], [new, 2], 4, 2, dh, 16, dtype, True)
    c["block_table"][0, 2] = -1
    table = c["block_table"].cpu().numpy()
    clean = atspeed_tree_attention(**c)
    for p, dim in ((50, 3), (99, 17)):                 # beside the bad page, and in the last context token
        c["v_cache"].view(-1, 2, dh)[table[0, p // 16] * 16 + p % 16, 1, dim] = poison
        got = atspeed_tree_attention(**c).float()[:new, 2:, dim]
        assert bool((got.isnan() if math.isnan(poison) else got == poison).all())
    got, clean = atspeed_tree_attention(**c).float(), clean.float()
    got[:new, 2:, 3] = clean[:new, 2:, 3]
    got[:new, 2:, 17] = clean[:new, 2:, 17]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (F32, 64)])
def test_attention_seen_infinite_values_reach_their_rows(dtype, dh):
    c = attention_case(12, [21, 5], [30, 8], 4, 2, dh, 16, dtype, True, levels=2)
    table, ctx = c["block_table"].cpu().numpy(), c["ctx"].cpu().numpy()
    p = int(ctx[0]) + 3                                # a root of the first tree
    slot = table[0, p // 16] * 16 + p % 16
    clean = atspeed_tree_attention(**c)
    c["v_cache"].view(-1, *c["v_cache"].shape[2:])[slot, 0, 5] = math.inf
    got = atspeed_tree_attention(**c).float().cpu()
    sees = ((c["mask"][:30, 0] >> 3) & 1).bool().cpu()
    assert 0 < int(sees.sum()) < 30
    assert bool((got[:30][sees][:, :2, 5] == math.inf).all())
    got[:30, :2, 5] = clean.float().cpu()[:30, :2, 5]
    assert torch.equal(got, clean.float().cpu())


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_attention_strides_scale_and_place(dtype, dh):
    """q out of a fused projection, head-major caches, q in place, another scale: same bits as the plain layout."""
    c = attention_case(21, [33, 100], [12, 50], 6, 2, dh, 32, dtype, True)
    scale = -0.37
    want = atspeed_tree_attention(**c, scale=scale)
    close_to_exact(c, want, None, scale)
    n = c["q"].shape[0]
    wide = torch.zeros((n, 10, dh), dtype=dtype, device=DEV)
    wide[:, 3:9] = c["q"]
    lay = dict(c, q=wide[:, 3:9], k_cache=c["k_cache"].transpose(1, 2).contiguous().transpose(1, 2),
               v_cache=torch.cat([c["v_cache"], c["v_cache"]], -1)[..., :dh])
    assert torch.equal(atspeed_tree_attention(**lay, scale=scale), want)
    out = atspeed_tree_attention(**lay, scale=scale, out=lay["q"])
    assert out.data_ptr() == lay["q"].data_ptr() and torch.equal(wide[:, 3:9], want)
    assert int(wide[:, :3].count_nonzero()) == 0 and int(wide[:, 9:].count_nonzero()) == 0


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (F32, 32)])
def test_attention_of_scale_zero_is_the_mean(dtype, dh):
    c = attention_case(23, [70, 3], [40, 2], 4, 2, dh, 16, dtype, True)
    close_to_exact(c, *atspeed_tree_attention(**c, scale=0.0, return_lse=True), scale=0.0)


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (F32, 64)])
@pytest.mark.parametrize("new", [1, 40])
def test_attention_stays_inside_for_nonsense_lengths(dtype, dh, new):
    """Row offsets, contexts and pages hold garbage: no access leaves the buffers, rows of sane requests are right."""
    c = attention_case(24, [100, 50, 3000], [new, new, new], 4, 2, dh, 16, dtype, True)
    want = atspeed_tree_attention(**c)
    rng = np.random.default_rng(3)
    for off in ([0, new, -5, 3 * new], [0, 2 ** 31 - 1, -2 ** 31, 7], [-9, new, 2 * new, 3 * new], [5, 4, 3, 2]):
        for ctx in (c["ctx"], ints([2 ** 31 - 1, -2 ** 31, 10 ** 9])):
            bad = dict(c, row_off=ints(off), ctx=ctx, block_table=ints(rng.integers(-2 ** 31, 2 ** 31, c["block_table"].shape)))
            atspeed_tree_attention(**bad)
            atspeed_tree_attention(**dict(bad, mask=None))
    got = atspeed_tree_attention(**dict(c, row_off=ints([0, new, 2 * new, -7])))
    assert torch.equal(got[:2 * new], want[:2 * new])


def test_attention_with_parts_in_a_graph():
    """A split context in two captured graphs that replay in turn: each equals its eager call."""
    cases = [attention_case(81 + i, [9000, 40, 2500], [5, 3, 6], 8, 2, 128, 16, BF16, True) for i in range(2)]
    want = [atspeed_tree_attention(**c, return_lse=True) for c in cases]
    torch.cuda.synchronize()
    graphs, got = [torch.cuda.CUDAGraph() for _ in cases], []
    for g, c in zip(graphs, cases):
        with torch.cuda.graph(g):
            got.append(atspeed_tree_attention(**c, return_lse=True))
    for _ in range(3):
        for g, x, w in zip(graphs, got, want):
            for t in x:
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(x[0], w[0]) and torch.equal(x[1], w[1])


def test_strides_of_dimensions_of_one_element_do_not_matter():
    c = attention_case(22, [20], [1], 1, 1, 64, 32, BF16, False)
    odd = lambda t, *s: torch.as_strided(t, t.shape, s)  # noqa: E731
    want = atspeed_tree_attention(**c)
    assert c["k_cache"].shape[2] == 1
    got = atspeed_tree_attention(**dict(c, q=odd(c["q"], 3, 5, 1), k_cache=odd(c["k_cache"], *c["k_cache"].stride()[:2], 7, 1)))
    assert torch.equal(got, want)
    k = torch.randn((1, 1, 64), device=DEV).to(BF16)
    a, b = (torch.zeros((4, 8, 1, 64), dtype=BF16, device=DEV) for _ in range(2))
    atspeed_kv_append(odd(k, 1, 3, 1), k, odd(a, 512, 64, 9, 1), b, ints([9]))
    assert torch.equal(a[1, 1], k[0]) and torch.equal(b, a)


def test_attention_leaves_other_rows_alone():
    c = attention_case(8, [40, 9], [7, 5], 4, 2, 128, 16, BF16, True, spare=6)
    out = torch.full_like(c["q"], 3.0)
    atspeed_tree_attention(**c, out=out)
    assert bool((out[12:] == 3.0).all())
    # a bound below a request's rows: the rows past it stay
    out = torch.full_like(c["q"], 3.0)
    want = atspeed_tree_attention(**c)
    atspeed_tree_attention(**dict(c, max_new=5), out=out)
    assert bool((out[5:7] == 3.0).all()) and torch.equal(out[:5], want[:5]) and torch.equal(out[7:12], want[7:12])


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (F32, 64)])
def test_attention_skips_bad_pages(dtype, dh):
    """Keys in pages outside the pool, and past the table, are not seen."""
    c = attention_case(31, [100, 90], [10, 70], 4, 2, dh, 16, dtype, True)
    c["block_table"][0, 2], c["block_table"][1, 0], c["block_table"][1, 6] = 2 ** 31 - 1, -5, c["k_cache"].shape[0]
    close_to_exact(c, *atspeed_tree_attention(**c, return_lse=True))
    c["block_table"] = c["block_table"][:, :5].contiguous()
    close_to_exact(c, *atspeed_tree_attention(**c, return_lse=True))


def test_attention_context_above_its_bound_is_read_whole():
    c = attention_case(41, [3000, 10], [4, 4], 8, 2, 128, 16, BF16, True)
    got = atspeed_tree_attention(**dict(c, max_ctx=100), return_lse=True)
    close_to_exact(c, *got)


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (F32, 64)])
def test_attention_is_repeatable(dtype, dh):
    c = attention_case(51, [4000, 700, 4000], [3, 3, 3], 8, 2, dh, 16, dtype, True)
    a, b = atspeed_tree_attention(**c), atspeed_tree_attention(**c)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,dh", TYPES)
@pytest.mark.parametrize("most", [1, 20, 40])
def test_attention_of_many_short_requests(dtype, dh, most):
    rng = np.random.default_rng(most)
    c = attention_case(62, rng.integers(0, 200, 40), rng.integers(0, most + 1, 40), 8, 8, dh, 16, dtype, True)
    close_to_exact(c, *atspeed_tree_attention(**c, return_lse=True))


@pytest.mark.parametrize("dtype,dh", TYPES)
@pytest.mark.parametrize("most", [60, 200])
@pytest.mark.parametrize("tree", [True, False])
def test_attention_of_many_requests_with_many_rows(dtype, dh, most, tree):
    """Launches that fill the GPU with tiles of 64 and 128 queries, last tiles of every size."""
    rng = np.random.default_rng(most)
    ctx, new = rng.integers(0, 90, 50), rng.integers(0, most + 1, 50)
    new[:4] = most, min(most, 129), min(most, 192), min(most, 65)
    c = attention_case(63, ctx, new, 8, 8, dh, 16, dtype, tree)
    close_to_exact(c, *atspeed_tree_attention(**c, return_lse=True))


@pytest.mark.parametrize("dtype,dh", [(BF16, 128), (BF16, 64), (F32, 32), (F32, 64)])
@pytest.mark.parametrize("B,most", [(5, 40), (64, 1), (70, 1), (70, 9), (130, 80)])
@pytest.mark.parametrize("tree", [True, False])
def test_attention_cuts_ragged_batches_into_even_pieces(dtype, dh, B, most, tree):
    """Long and short contexts and requests without rows, in batches of more requests than a wave has lanes."""
    rng = np.random.default_rng(B + most)
    ctx, new = rng.integers(0, 3000, B), rng.integers(0, most + 1, B)
    ctx[1], ctx[-1], new[0], new[-1] = 0, 3000, 0, most
    c = attention_case(61, ctx, new, 2, 1, dh, 16, dtype, tree)
    close_to_exact(c, *atspeed_tree_attention(**c, return_lse=True))


# ---------------------------------------------------------------- logit rules

def rules_case(seed, B, new, cols, dtype, tree=True, hist=50, states=5, n_bias=2):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    new = np.array(new if len(np.shape(new)) else [new] * B)
    n, base, width = int(new.sum()), 500, max(1, int(np.max(new)))
    tok = lambda *s: ints(rng.integers(base - 3, base + min(cols, 40) + 3, s))  # noqa: E731
    f = lambda lo, hi: torch.from_numpy(rng.uniform(lo, hi, B).astype(np.float32)).to(DEV)  # noqa: E731
    parents = np.stack([ref.tree_parents(rng, int(m), 3, width) for m in new])
    allowed = rng.integers(-2 ** 31, 2 ** 31, (states, (cols + 31) // 32))
    return dict(logits=(torch.randn((n, cols), generator=g, device=DEV) * 3).to(dtype),
                row_off=ints(np.concatenate([[0], np.cumsum(new)])), token_base=base, history=tok(B, hist),
                hist_len=ints(rng.integers(-2, hist + 4, B)), repetition=f(0.7, 1.6), frequency=f(-0.3, 0.6),
                presence=f(-0.2, 0.5), temperature=f(0.3, 1.8),
                bias=torch.randn((n_bias, cols), generator=g, device=DEV), bias_index=ints(rng.integers(-1, n_bias + 1, B)),
                allowed=ints(allowed), state=ints(rng.integers(-1, states + 1, n)),
                mask=mask_of(parents, new) if tree else None, node_token=tok(B, width))


def check_rules(c, got=None, mask_value=-math.inf):
    """fp32: at most ten roundings of 2^-24 of what is added up (division, product, two sums, bias, division)."""
    got = atspeed_logit_rules(**c, mask_value=mask_value) if got is None else got
    want, size = ref.logit_rules(**c, mask_value=mask_value)
    live = int(c["row_off"][-1])
    got, want, size = got.cpu().double()[:live], want[:live], size[:live]
    same = (got == want) | (got.isnan() & want.isnan())
    off = (got - want).abs()
    assert bool((same | (off <= 10 * 2.0 ** -24 * size)).all())
    return got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1, 5, 31, 64, 257, 1000, 1024, 1025, 4096, 5001, 9000])
@pytest.mark.parametrize("tree", [True, False])
def test_rules_columns(dtype, cols, tree):
    check_rules(rules_case(cols, 4, [3, 0, 1, 6], cols, dtype, tree))


PARTS = ("history", "node_token", "repetition", "frequency", "presence", "temperature", "bias", "bias_index", "allowed")


@pytest.mark.parametrize("without", [()] + [(p,) for p in PARTS] + [PARTS[:2], PARTS[2:5], PARTS])
def test_rules_parts_left_out(without):
    c = rules_case(3, 3, [2, 5, 1], 300, F32)
    for p in without:
        c[p] = None
    if c["history"] is None:
        c["hist_len"] = None
    if c["allowed"] is None:
        c["state"] = None
    got = check_rules(c)
    if without == PARTS:
        assert torch.equal(got, c["logits"].cpu().double())


def test_rules_long_histories_and_many_requests():
    check_rules(rules_case(6, 300, 1, 700, BF16, False, hist=3000))
    check_rules(rules_case(7, 1024, 1, 33, F32, False, hist=2))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [8001, 8192])
def test_rules_many_long_rows(dtype, cols):
    check_rules(rules_case(6, 300, [1] * 300, cols, dtype, False))


def test_rules_wide_trees():
    check_rules(rules_case(8, 2, [130, 70], 200, F32))


@pytest.mark.parametrize("value", [-math.inf, -3.0e38, 0.0])
def test_rules_masked_columns_hold_the_mask_value(value):
    """NaN and infinities in masked columns go; in allowed ones they stay."""
    c = rules_case(9, 2, [4, 4], 100, F32)
    c["logits"][:, ::3], c["logits"][:, 1::3] = math.nan, -math.inf
    c["logits"][0, 2::3] = math.inf
    got = check_rules(c, mask_value=value)
    s = c["state"].cpu().numpy()
    a = c["allowed"].cpu().numpy()
    for r in range(8):
        if s[r] >= 0:
            ok = [s[r] < 5 and (int(a[s[r], v // 32]) >> (v % 32)) & 1 == 1 for v in range(100)]
            assert all(float(got[r, v]) == float(np.float32(value)) for v in range(100) if not ok[v])


def test_rules_in_place_strided_and_scattered():
    c = rules_case(10, 3, [2, 4, 3], 203, F32)
    want = atspeed_logit_rules(**c)
    wide = torch.zeros((9, 230), device=DEV)
    wide[:, 11:214] = c["logits"]
    moved = dict(c, logits=wide[:, 11:214])
    assert torch.equal(atspeed_logit_rules(**moved), want)
    out = torch.full((4, 5, 203), 7.0, device=DEV)
    rows = ints([0, 3, -1, 19, 7, 8, 20, 2, 11])
    atspeed_logit_rules(**moved, out=out, out_row=rows)
    flat, kept = out.view(20, 203), [r for r in rows.tolist() if 0 <= r < 20]
    for r, o in enumerate(rows.tolist()):
        if 0 <= o < 20:
            assert torch.equal(flat[o], want[r])
    assert bool((flat[[i for i in range(20) if i not in kept]] == 7.0).all())
    got = atspeed_logit_rules(**moved, out=moved["logits"])
    assert torch.equal(got, want) and torch.equal(wide[:, 11:214], want)
    assert int(wide[:, :11].count_nonzero()) == 0 and int(wide[:, 214:].count_nonzero()) == 0


def test_rules_with_a_state_for_each_request():
    c = rules_case(14, 4, [2, 0, 3, 1], 300, BF16)
    of = torch.tensor([2, -1, 7, 0], dtype=torch.int32, device=DEV)      # one set, none, one past the end, one set
    rows = of[torch.tensor([0, 0, 2, 2, 2, 3], device=DEV)].contiguous()
    want = atspeed_logit_rules(**dict(c, state=rows))
    assert torch.equal(atspeed_logit_rules(**dict(c, state=of), state_by_request=True), want)
    assert bool((want[2:5] == -math.inf).all())


def test_rules_stay_inside_for_nonsense_indices():
    c = rules_case(15, 3, [2, 3, 1], 90, F32)
    rng = np.random.default_rng(1)
    junk = lambda t: ints(rng.integers(-2 ** 31, 2 ** 31, t.shape))  # noqa: E731
    names = ("row_off", "history", "hist_len", "bias_index", "state", "node_token")
    for n in names:
        atspeed_logit_rules(**dict(c, **{n: junk(c[n])}))
    out = torch.full((6, 90), 5.0, device=DEV)
    atspeed_logit_rules(**dict(c, **{n: junk(c[n]) for n in names}), out=out, out_row=junk(c["state"]))
    assert torch.equal(out, torch.full_like(out, 5.0))
    check_rules(c)


def test_rules_rows_behind_the_last_request_stay():
    c = rules_case(12, 2, [3, 2], 64, F32)
    out = torch.full((5, 64), 9.0, device=DEV)
    c["row_off"] = ints([0, 3, 3])
    got = atspeed_logit_rules(**c, out=out)
    assert bool((got[3:] == 9.0).all())


# ---------------------------------------------------------------- streams, graphs

def test_operators_on_another_stream_and_in_a_graph():
    """One step captured and replayed over new lengths and inputs equals the eager calls, replay after replay."""
    rng = np.random.default_rng(2)
    g = torch.Generator(device=DEV).manual_seed(2)
    B, heads, kv, dh, width, cols = 6, 8, 2, 128, 20, 500

    def inputs(step):
        new = rng.integers(0, width + 1, B)
        parent = np.stack([ref.tree_parents(rng, int(m), 3, width) for m in new])
        r = lambda *s: torch.randn(s, generator=g, device=DEV).to(BF16)  # noqa: E731
        return dict(keep=ints(rng.integers(0, 60, B) * (step > 0)), add=ints(new), parent=ints(parent),
                    q=r(B * width, heads, dh), k=r(B * width, kv, dh), v=r(B * width, kv, dh),
                    logits=torch.randn((B * width, cols), generator=g, device=DEV),
                    token=ints(rng.integers(0, cols, (B, width))))

    def state():
        s = dict(held=torch.full((B,), 60, dtype=torch.int32, device=DEV), table=ints(np.arange(B * 10).reshape(B, 10)),
                 free=ints(np.arange(B * 10, B * 10 + 40)), n_free=ints([40]))
        s["free"] = torch.cat([s["free"], torch.full((60,), -1, dtype=torch.int32, device=DEV)])
        gg = torch.Generator(device=DEV).manual_seed(7)
        s["kc"], s["vc"] = (torch.randn((100, 8, kv, dh), generator=gg, device=DEV).to(BF16) for _ in range(2))
        return s

    def step(s, x):
        p = atspeed_page_plan(s["held"], x["keep"], x["add"], s["table"], s["free"], s["n_free"], 8, B * width, x["parent"])
        atspeed_kv_append(x["k"], x["v"], s["kc"], s["vc"], p.slot)
        out = atspeed_tree_attention(x["q"], s["kc"], s["vc"], s["table"], p.row_off, p.ctx, 60, width, mask=p.mask,
                                     out=torch.zeros_like(x["q"]))
        z = atspeed_logit_rules(x["logits"], p.row_off, mask=p.mask, node_token=x["token"],
                                repetition=torch.full((B,), 1.3, device=DEV), out=torch.zeros_like(x["logits"]))
        s["held"].copy_(p.length)
        s["n_free"].copy_(p.n_free)
        return p, out, z

    eager, graphed, xs = state(), state(), [inputs(i) for i in range(5)]
    hold = {k: v.clone() for k, v in xs[0].items()}
    side = torch.cuda.Stream(device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(state(), hold)                            # warm up on the other stream
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(graphed, hold)
    for x in xs:
        for k in hold:
            hold[k].copy_(x[k])
        graph.replay()
        want = step(eager, x)
        torch.cuda.synchronize()
        n = int(want[0].row_off[-1])
        for a, b in zip(got[0], want[0]):
            assert torch.equal(a, b)
        assert torch.equal(got[1][:n], want[1][:n]) and torch.equal(got[2][:n], want[2][:n])
        for k in ("held", "table", "n_free", "kc", "vc"):
            assert torch.equal(graphed[k], eager[k]), k


def test_two_calls_at_once_on_two_streams():
    cases = [attention_case(61 + i, [5000, 300], [2, 30], 8, 2, 128, 16, BF16, True) for i in range(2)]
    want = [atspeed_tree_attention(**c) for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(device=DEV) for _ in cases], [[], []]
    for _ in range(4):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                got[i].append(atspeed_tree_attention(**c))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_calls_from_two_threads():
    cases = [attention_case(64 + i, [5000, 300], [2, 30], 8, 2, 128, 16, BF16, True) for i in range(2)]
    want = [atspeed_tree_attention(**c, return_lse=True) for c in cases]
    torch.cuda.synchronize()
    got = [[], []]

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream(device=DEV)):
            for _ in range(20):
                got[i].append(atspeed_tree_attention(**cases[i], return_lse=True))
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        assert len(got[i]) == 20 and all(torch.equal(x, y) for r in got[i] for x, y in zip(r, want[i]))


def test_calls_keep_no_reference():
    c = attention_case(66, [5000, 30], [2, 3], 8, 2, 128, 16, BF16, True)
    r = rules_case(2, 2, [1, 1], 50, F32)
    out, z = torch.empty_like(c["q"]), torch.empty((2, 50), device=DEV)
    held = [*c.values(), *r.values(), out, z]
    refused = dict(c, ctx=c["ctx"].long())

    def calls():
        for _ in range(5):
            assert atspeed_tree_attention(**c, out=out) is out and atspeed_logit_rules(**r, out=z) is z
            atspeed_tree_attention(**c, return_lse=True)
            try:
                atspeed_tree_attention(**refused)
                raise AssertionError("not refused")
            except ValueError:
                pass

    calls()
    before = [sys.getrefcount(t) for t in held if isinstance(t, torch.Tensor)]
    torch.cuda.synchronize()
    used = torch.cuda.memory_allocated()
    calls()
    assert [sys.getrefcount(t) for t in held if isinstance(t, torch.Tensor)] == before
    assert torch.cuda.memory_allocated() == used


# ---------------------------------------------------------------- refusals that reach the tensors

def test_refusals_of_tensors():
    c = attention_case(71, [5], [3], 4, 2, 128, 16, BF16, True)
    bad = [dict(q=c["q"].float()), dict(q=c["q"].cpu()), dict(q=c["q"][:, :, ::2]), dict(k_cache=c["k_cache"].float()),
           dict(ctx=c["ctx"].long()), dict(ctx=c["ctx"].cpu()), dict(row_off=c["row_off"][:1]),
           dict(mask=c["mask"][:2]), dict(block_table=c["block_table"].t())]
    for kw in bad:
        with pytest.raises(ValueError):
            atspeed_tree_attention(**dict(c, **kw))
    with pytest.raises(ValueError):
        atspeed_tree_attention(**dict(c, max_ctx=2 ** 40))
    r = rules_case(1, 2, [1, 1], 50, F32)
    for kw in (dict(logits=r["logits"].double()), dict(state=r["state"][:1]), dict(bias=r["bias"][:, :49]),
               dict(allowed=r["allowed"][:, :1]), dict(history=r["history"].long()), dict(out_row=ints([0, 1]))):
        with pytest.raises(ValueError):
            atspeed_logit_rules(**dict(r, **kw))

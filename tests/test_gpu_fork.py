"""Forked pages, page copies and accepted paths against plain implementations."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import _beam_reference as ref  # noqa: E402
from paper_2410_05165_amd.binding import AtspeedError  # noqa: E402
from paper_2410_05165_amd.paged import (PagedKV, atspeed_kv_compact, atspeed_page_copy,  # noqa: E402
                                        atspeed_page_fork)

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
OUT = ("length", "refused", "copy_src", "copy_dst", "copy_len")


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


# ---------------------------------------------------------------- page tables

def fork_case(rng, users, beams, page, most, spare=None, bad=False):
    """Users whose beams share their first pages; consistent holders and free list."""
    B = users * beams
    table, held = np.full((B, most), -1), np.zeros(B, np.int64)
    pool = B * most + 3
    order = list(rng.permutation(pool))
    shared = np.zeros(pool, np.int64)
    for u in range(users):
        joint = int(rng.integers(0, most + 1))
        pages = [order.pop() for _ in range(joint)]
        for j in range(u * beams, (u + 1) * beams):
            if rng.random() < 0.1:
                continue                                       # an empty row
            held[j] = rng.integers(0, most * page + 1) if rng.random() < 0.3 else min(most * page, joint * page + rng.integers(0, 2 * page))
            need = -(-int(held[j]) // page)
            for c in range(need):
                table[j, c] = pages[c] if c < joint else order.pop()
                shared[table[j, c]] += 1
    shared = np.maximum(shared - 1, 0)
    n_free = len(order) if spare is None else min(spare, len(order))
    free = np.full(pool, -1)
    free[:n_free] = order[:n_free]
    src = rng.integers(0, beams, B) + np.repeat(np.arange(users), beams) * beams
    src[rng.random(B) < 0.15] = -1
    src[rng.random(B) < 0.1] = rng.integers(0, B)
    keep = np.where(rng.random(B) < 0.6, held[np.maximum(src, 0)], rng.integers(0, held[np.maximum(src, 0)] + 1))
    if bad:
        for j in range(B):
            what = rng.integers(0, 10)
            if what == 0:
                src[j] = B
            elif what == 1:
                src[j] = -2
            elif what == 2:
                keep[j] = held[max(src[j], 0)] + 1
            elif what == 3:
                keep[j] = -1
            elif what == 4:
                held[j] = -3
            elif what == 5:
                held[j] = most * page + 1
            elif what == 6:
                table[j, rng.integers(0, most)] = pool + 5
    return held, keep, table, free, n_free, shared, src


def check_fork(c, page, with_src=True, with_keep=True):
    held, keep, table, free, n_free, shared, src = c
    keep, src = keep if with_keep else None, src if with_src else None
    t, f, n, s = ints(table), ints(free), ints([n_free]), ints(shared)
    got = atspeed_page_fork(ints(held), None if keep is None else ints(keep), t, f, n, s, page,
                            src=None if src is None else ints(src))
    want = ref.fork(held, keep, table, free, n_free, shared, page, src)
    for name in OUT:
        assert getattr(got, name).tolist() == want[name], name
    assert n.tolist() == [want["n_free"]] and s.tolist() == want["shared"]
    for g, w in zip(f.tolist(), want["free"]):
        assert w is None or g == w
    for g, w in zip(t.tolist(), want["table"]):
        assert all(b is None or a == b for a, b in zip(g, w))
    return got


@pytest.mark.parametrize("users,beams,page,most", [(1, 1, 1, 1), (1, 10, 16, 6), (3, 4, 8, 5), (32, 10, 16, 9), (1024, 1, 4, 3),
                                                   (20, 50, 64, 4), (2, 5, 16, 300), (1, 1000, 2, 40)])
@pytest.mark.parametrize("seed", range(3))
def test_fork_equals_the_sequential_one(users, beams, page, most, seed):
    rng = np.random.default_rng(100 * users + 10 * beams + seed)
    c = fork_case(rng, users, beams, page, most)
    check_fork(c, page)
    check_fork(c, page, with_keep=False)


@pytest.mark.parametrize("seed", range(6))
def test_dropping_tokens_without_a_fork(seed):
    c = fork_case(np.random.default_rng(seed), 6, 5, 8, 6)
    held, keep = c[0], np.random.default_rng(seed + 50).integers(0, c[0] + 1)
    check_fork((held, keep) + c[2:], 8, with_src=False)
    check_fork(c, 8, with_src=False, with_keep=False)        # nothing changes


@pytest.mark.parametrize("rows,pool", [(3, 5), (3, 700), (200, 600)])
def test_pages_held_more_often_than_counted(rows, pool):
    """They are counted below -1: taken once, or back once, and the pages behind keep their places in the free list."""
    table = np.full((rows, 2), -1)
    table[:, 0] = 0
    table[0, 1], table[1, 1] = pool - 1, pool - 1            # dropped by both, in the pool's last piece
    held = np.full(rows, 4)
    held[:2] = 8
    free = np.full(pool, -1)
    shared = np.zeros(pool, np.int64)
    src = np.full(rows, -1)
    src[2] = 2                                               # goes on with part of page 0, which is its own now
    keep = np.where(src < 0, 0, 3)
    for n_free in (0, 1):
        free[:n_free] = 1
        got = check_fork((held, keep, table, free, n_free, shared, src), 4)
        assert got.copy_dst.tolist() == [-1] * rows and got.length.tolist() == [3 if j == 2 else 0 for j in range(rows)]


@pytest.mark.parametrize("rows,most,pool", [(8, 5, 60), (300, 5, 1500), (300, 5, 400)])
@pytest.mark.parametrize("seed", range(4))
def test_whatever_shared_holds_nothing_leaves_its_buffer(rows, most, pool, seed):
    rng = np.random.default_rng(seed)
    page, edge = 4, 64
    held = rng.integers(0, most * page + 1, rows)
    src = rng.integers(-1, rows, rows)
    keep = rng.integers(0, np.where(src < 0, 0, held[np.maximum(src, 0)]) + 1)
    shared = rng.integers(-3, 4, pool)
    shared[rng.integers(0, pool, 3)] = [-2**31, 2**31 - 1, -2**31 + 1]
    table = rng.integers(0, pool, (rows, most))
    n_free = int(rng.integers(0, pool + 1))

    def inside(a):
        whole = torch.full((a.size + 2 * edge,), -77, dtype=torch.int32, device=DEV)
        whole[edge:edge + a.size] = ints(a).view(-1)
        return whole, whole[edge:edge + a.size].view(a.shape)

    (t_all, t), (f_all, f), (s_all, s) = inside(table), inside(rng.permutation(pool)), inside(shared)
    n_all, n = inside(np.array([n_free]))
    got = atspeed_page_fork(ints(held), ints(keep), t, f, n, s, page, src=ints(src))
    for whole, size in ((t_all, rows * most), (f_all, pool), (s_all, pool), (n_all, 1)):
        assert bool((whole[:edge] == -77).all()) and bool((whole[edge + size:] == -77).all())
    left = int(n)
    assert 0 <= left <= pool and all(0 <= p < pool for p in f.tolist()) and all(0 <= p < pool for p in t.view(-1).tolist())
    for j, (length, dst, size) in enumerate(zip(got.length.tolist(), got.copy_dst.tolist(), got.copy_len.tolist())):
        assert 0 <= length <= most * page and -1 <= dst < pool and 0 <= size < page


@pytest.mark.parametrize("seed", range(12))
def test_fork_with_too_few_pages_and_malformed_rows(seed):
    rng = np.random.default_rng(seed)
    check_fork(fork_case(rng, 8, 6, 8, 5, spare=int(rng.integers(0, 12)), bad=seed % 2 == 1), 8)


def test_every_last_page_is_refused_without_pages():
    """Full pages stay, the tokens of the last one are dropped."""
    held, table = np.array([20, 20, 20]), np.array([[0, 1, 2], [3, 4, 5], [6, 7, 8]])
    c = (held, held, table, np.full(9, -1), 0, np.zeros(9, int), np.array([0, 0, 0]))
    got = check_fork(c, 8)
    # 3 .. 8 come free: two of them are copies of page 2
    assert got.refused.tolist() == [0, 0, 0] and got.copy_dst.tolist() == [-1, 8, 7]
    c = (np.array([20, 20, 0]), np.array([20, 20, 0]), np.array([[0, 1, 2], [0, 1, 2], [-1, -1, -1]]), np.full(3, -1), 0,
         np.array([1, 1, 1]), np.array([0, 1, -1]))
    got = check_fork(c, 8)
    assert got.refused.tolist() == [0, 1, 0] and got.length.tolist() == [20, 16, 0]


def test_a_page_that_the_caller_keeps_is_never_taken_or_freed():
    held, table = np.array([12, 12]), np.array([[0, 1], [0, 2]])
    shared = np.array([1, 1, 0, 0, 0])                       # page 1: row 0 and the caller
    c = (held, held, table, np.array([3, 4, -1, -1, -1]), 2, shared, np.array([0, 0]))
    got = check_fork(c, 8)
    assert got.copy_src.tolist() == [1, 1] and set(got.copy_dst.tolist()) <= {2, 3, 4}


def test_fork_survives_nonsense_state():
    rng = np.random.default_rng(0)
    wild = lambda *s: rng.integers(-2 ** 31, 2 ** 31, s)  # noqa: E731
    for _ in range(6):
        t, f, n, s = ints(wild(9, 5)), ints(wild(30)), ints(wild(1)), ints(rng.integers(-5, 5, 30))
        got = atspeed_page_fork(ints(wild(9)), ints(wild(9)), t, f, n, s, 8, src=ints(wild(9)))
        some = atspeed_page_fork(ints(rng.integers(0, 41, 9)), ints(rng.integers(0, 41, 9)), t, f, n, s, 8,
                                 src=ints(rng.integers(-1, 9, 9)))
        torch.cuda.synchronize()
        assert 0 <= int(n[0]) <= 30 and bool((got.refused == 2).any()) and bool((some.length <= 40).all())


def test_large_pools():
    """Pools whose pieces are longer than a workgroup's step."""
    rng = np.random.default_rng(4)
    held, keep, table, free, n_free, shared, src = fork_case(rng, 4, 6, 16, 7)
    pool = 1_500_000
    move = np.sort(rng.choice(pool, len(shared), replace=False))
    big = np.zeros(pool, np.int64)
    big[move] = shared
    wide = np.full(pool, -1)
    wide[:n_free] = move[free[:n_free]]
    check_fork((held, keep, np.where(table >= 0, move[np.maximum(table, 0)], -1), wide, n_free, big, src), 16)


# ---------------------------------------------------------------- moving tokens

def caches(seed, layers, pool, page, heads, dh, dtype):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [torch.randn((layers, pool, page, heads, dh), generator=g, device=DEV).to(dtype) for _ in range(2)]


LAYOUTS = [(F32, 32, 4), (F32, 64, 1), (F32, 128, 3), (BF16, 64, 2), (BF16, 128, 8), (BF16, 128, 40)]


@pytest.mark.parametrize("dtype,dh,heads", LAYOUTS)
@pytest.mark.parametrize("page,layers", [(1, 3), (16, 1), (64, 5)])
def test_page_copies(dtype, dh, heads, page, layers):
    rng = np.random.default_rng(dh + page)
    n = 9
    k, v = caches(page, layers, 2 * n + 2, page, heads, dh, dtype)
    src, dst, length = rng.integers(0, n, n), rng.permutation(n) + n, rng.integers(0, page + 1, n)
    src[1], dst[2], src[3], dst[4], length[5], length[6] = -1, -1, 2 * n + 2, 2 ** 30, page + 100, -4
    wk, wv = k.clone(), v.clone()
    for a, b, m in zip(src, dst, length):
        if 0 <= a < 2 * n + 2 and 0 <= b < 2 * n + 2 and m > 0:
            for w, x in ((wk, k), (wv, v)):
                w[:, b, :m] = x[:, a, :m]
    atspeed_page_copy(k, v, ints(src), ints(dst), ints(length))
    assert torch.equal(k, wk) and torch.equal(v, wv)
    one = [x[-1].clone() for x in (k, v)]                     # caches of one layer, four dimensions
    atspeed_page_copy(one[0], one[1], ints([0]), ints([2 * n + 1]), ints([page]))
    assert torch.equal(one[0][2 * n + 1], k[-1, 0]) and torch.equal(one[1][2 * n + 1], v[-1, 0])


def paths_case(rng, B, page, most, width, P):
    ctx = rng.integers(0, most * page - width + 1, B)
    table = rng.permutation(B * most).reshape(B, most)
    n_path = rng.integers(0, P + 1, B)
    path = np.full((B, P), -7)
    for b in range(B):
        path[b, :n_path[b]] = np.sort(rng.choice(width, n_path[b], replace=False))
    return ctx, table, path, n_path


def compacted(x, page, ctx, table, path, n_path):
    w = x.clone()
    for b in range(len(ctx)):
        for i in range(n_path[b]):
            a, to = ctx[b] + path[b, i], ctx[b] + i
            w[:, table[b, to // page], to % page] = x[:, table[b, a // page], a % page]
    return w


@pytest.mark.parametrize("dtype,dh,heads", LAYOUTS)
@pytest.mark.parametrize("page,P", [(1, 1), (4, 4), (16, 8), (64, 40)])
def test_paths_move_together(dtype, dh, heads, page, P):
    rng = np.random.default_rng(page + dh)
    width = max(P, 45)
    B, most = 7, -(-60 // page) + -(-width // page)
    c = paths_case(rng, B, page, most, width, P)
    k, v = caches(page + 1, 3, B * most, page, heads, dh, dtype)
    want = [compacted(x, page, *c) for x in (k, v)]
    atspeed_kv_compact(k, v, ints(c[1]), ints(c[0]), ints(c[2]), ints(c[3]))
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_long_paths():
    rng = np.random.default_rng(9)
    c = paths_case(rng, 3, 16, 320, 5000, 4096)
    c[3][:] = [4096, 4095, 0]
    for b in range(2):
        c[2][b, :c[3][b]] = np.sort(rng.choice(5000, c[3][b], replace=False))
    k, v = caches(5, 1, 960, 16, 1, 64, BF16)
    want = [compacted(x, 16, *c) for x in (k, v)]
    atspeed_kv_compact(k, v, ints(c[1]), ints(c[0]), ints(c[2]), ints(c[3]))
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_malformed_paths_move_nothing():
    """Each bad request stays as it was, its neighbours move."""
    page, most = 8, 5
    table = np.arange(10 * most).reshape(10, most)
    ctx = np.full(10, 9)
    path = np.tile([1, 3, 6, 8], (10, 1))
    n_path = np.full(10, 4)
    path[1, 2] = 3                                            # twice the same
    path[2, 1] = 0                                            # descending
    path[3, 0] = -1
    ctx[4] = -1
    n_path[5], n_path[6] = 5, -2
    path[7, 3] = 40                                           # past the table
    table[8, 2] = 1000                                        # a bad page
    ctx[9] = 2 ** 31 - 1
    k, v = caches(3, 2, 50, page, 2, 64, BF16)
    want = []
    for x in (k, v):
        good = [0]
        want.append(compacted(x, page, ctx[good], table[good], path[good], n_path[good]))
    atspeed_kv_compact(k, v, ints(table), ints(ctx), ints(path), ints(n_path))
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


@pytest.mark.parametrize("what", ["copy", "compact"])
def test_strided_caches(what):
    """Layers, pages, tokens and heads with room between them that stays as it was; heads first."""
    big = [torch.zeros((3, 12, 2, 18, 3, 96), dtype=F32, device=DEV) for _ in range(2)]
    for b in big:
        b.uniform_(-1, 1, generator=torch.Generator(device=DEV).manual_seed(1))
    view = lambda b: b[:, :, 0, 1:17, :2, 16:80]                        # noqa: E731  [3, 12, 16, 2, 64]
    k, v = view(big[0]), view(big[1]).clone().transpose(2, 3).contiguous().transpose(2, 3)     # v: heads before tokens
    before, kk, vv = big[0].clone(), k.clone(), v.clone()
    if what == "copy":
        args = (ints([0, 3]), ints([5, 7]), ints([9, 16]))
        atspeed_page_copy(kk, vv, *args)
        atspeed_page_copy(k, v, *args)
    else:
        args = (ints([[0, 1], [2, 3]]), ints([10, 3]), ints([[1, 4, 5], [0, 2, 9]]), ints([3, 3]))
        atspeed_kv_compact(kk, vv, *args)
        atspeed_kv_compact(k, v, *args)
    assert torch.equal(k, kk) and torch.equal(v, vv) and not torch.equal(kk, view(before))
    view(before).copy_(kk)
    assert torch.equal(big[0], before)


def test_moves_past_32_bits_of_elements():
    """A layer of more than 2^32 bytes, pages on both sides."""
    shape = (2, 70_000, 16, 16, 128)                          # 2.3e9 elements a layer
    k, v = (torch.zeros(shape, dtype=BF16, device=DEV) for _ in range(2))
    k[:, 2], v[:, 69_999] = 3.0, 5.0
    v[:, 2] = 4.0
    atspeed_page_copy(k, v, ints([2]), ints([69_998]), ints([7]))
    assert bool((k[:, 69_998, :7] == 3).all()) and bool((v[:, 69_998, :7] == 4).all())
    assert not bool(k[:, 69_998, 7:].any())
    atspeed_kv_compact(k, v, ints([[2, 69_999]]), ints([5]), ints([[20]]), ints([1]))
    assert bool((v[:, 2, 5] == 5).all()) and bool((k[:, 2, 5] == 0).all()) and bool((k[:, 2, 4] == 3).all())


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("seed", range(3))
def test_caches_of_forked_rows_hold_their_own_tokens(seed):
    """Random forks, growth and drops of PagedKV rows: every row reads the tokens that it was given."""
    rng = np.random.default_rng(seed)
    B, page, most = 8, 4, 32
    kv = PagedKV(2, 60, page, 1, 64, B, most, dtype=F32, share=True)
    texts, number = [[] for _ in range(B)], 1
    for step in range(25):
        src = rng.integers(-1, B, B) if step % 3 else np.arange(B)
        keep = np.array([0 if s < 0 else int(rng.integers(max(0, len(texts[s]) - 5), len(texts[s]) + 1)) for s in src])
        add = np.minimum(rng.integers(0, 6, B), most - keep)
        p = kv.plan(ints(keep), ints(add), 48, src=ints(src))
        refused = p.refused.tolist()
        rows = torch.zeros((48, 1, 64), device=DEV)
        new, at = [], 0
        length = kv.length.tolist()
        for j in range(B):
            mine = (texts[src[j]] if src[j] >= 0 else [])[:keep[j]]
            for _ in range(add[j]):
                rows[at] = number
                if not refused[j]:
                    mine = mine + [number]
                number, at = number + 1, at + 1
            new.append(mine[:length[j]])
            assert len(new[j]) == length[j] and (refused[j] or length[j] == keep[j] + add[j])
        texts = new
        for layer in range(2):
            kv.append(layer, p, rows, -rows)
        table = kv.block_table.cpu().numpy()
        holders = np.zeros(60, int)
        for j in range(B):
            for c in range(-(-length[j] // page)):
                holders[table[j, c]] += 1
            for t, want in enumerate(texts[j]):
                at = (1, table[j, t // page], t % page, 0, 5)
                assert float(kv.k[at]) == want and float(kv.v[at]) == -want, (step, j, t)
        n = int(kv.n_free)
        assert sorted(kv.free_pages[:n].tolist()) == [q for q in range(60) if not holders[q]]
        assert kv.shared.tolist() == [max(h - 1, 0) for h in holders]


def test_forks_and_moves_in_a_graph():
    """A step that forks, copies, plans, appends and compacts, captured once and replayed, goes on as the eager one."""
    rng = np.random.default_rng(3)
    B, page, most = 6, 4, 40

    def make():
        return PagedKV(2, 90, page, 2, 64, B, most, dtype=BF16, share=True)

    def step(kv, x):
        p = kv.plan(x["keep"], x["add"], B * 5, src=x["src"])
        for layer in range(2):
            kv.append(layer, p, x["k"], x["v"])
        return kv.compact(p, x["path"], x["n_path"])

    def inputs(length):
        src = rng.integers(-1, B, B)
        keep = np.array([0 if s < 0 else rng.integers(max(0, length[s] - 3), length[s] + 1) for s in src])
        add = np.minimum(rng.integers(1, 6, B), most - keep)
        n_path = rng.integers(0, np.minimum(add, 3) + 1)
        path = np.full((B, 3), -1)
        for b in range(B):
            path[b, :n_path[b]] = np.sort(rng.choice(add[b], n_path[b], replace=False))
        r = lambda: torch.randn((B * 5, 2, 64), device=DEV).to(BF16)  # noqa: E731
        return dict(src=ints(src), keep=ints(keep), add=ints(add), path=ints(path), n_path=ints(n_path), k=r(), v=r())

    eager, graphed = make(), make()
    hold = inputs(np.zeros(B, int))
    side = torch.cuda.Stream(device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm = make()
        step(warm, hold)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(graphed, hold)
    length = np.zeros(B, int)
    for _ in range(8):
        x = inputs(length)
        for name in hold:
            hold[name].copy_(x[name])
        graph.replay()
        want = step(eager, x)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        for name in ("length", "block_table", "n_free", "shared", "k", "v"):
            assert torch.equal(getattr(graphed, name), getattr(eager, name)), name
        n = int(eager.n_free)
        assert torch.equal(graphed.free_pages[:n], eager.free_pages[:n])
        length = eager.length.cpu().numpy()


def test_refusals():
    kv = PagedKV(2, 6, 4, 1, 64, 2, 8)
    with pytest.raises(ValueError, match="share"):
        kv.plan(ints([0, 0]), ints([1, 1]), 4, src=ints([0, 0]))
    c, i = torch.zeros((2, 6, 4, 1, 64), device=DEV), ints([0, 1])
    t, f, n = ints(np.zeros((2, 3))), ints(np.zeros(6)), ints([6])
    for call in (lambda: atspeed_page_fork(i, i, t, f, n, ints([0]), 4),
                 lambda: atspeed_page_fork(i, i.long(), t, f, n, f, 4),
                 lambda: atspeed_page_fork(i, i, t[0], f, n, f, 4),
                 lambda: atspeed_page_fork(ints([1]), i, t, f, n, f, 4),
                 lambda: atspeed_page_copy(c, c.bfloat16(), i, i, i), lambda: atspeed_page_copy(c[0, 0], c[0, 0], i, i, i),
                 lambda: atspeed_page_copy(c, c, i, ints([1]), i), lambda: atspeed_page_copy(c.half(), c.half(), i, i, i),
                 lambda: atspeed_page_copy(c, c[:1], i, i, i),
                 lambda: atspeed_kv_compact(c, c, t, i, i, i), lambda: atspeed_kv_compact(c, c, t, i, t.long(), i),
                 lambda: atspeed_kv_compact(c, c, t, ints([0]), t, i)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: atspeed_page_fork(i, i, t, f, n, f, 5),
                 lambda: atspeed_page_copy(c[..., :32].contiguous().bfloat16(), c[..., :32].contiguous().bfloat16(), i, i, i),
                 lambda: atspeed_kv_compact(c, c, t, i, ints(np.zeros((2, 5000))), i)):
        with pytest.raises(AtspeedError):
            call()
    leaf = torch.ones_like(c, requires_grad=True)
    square = (leaf * c).sum()                                 # saves c
    atspeed_page_copy(c, c.clone(), i, i, i)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        square.backward()

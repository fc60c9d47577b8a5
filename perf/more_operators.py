"""Measured cases of the operators around a caller's own target and draft: the selection of the
next beams over beams and vocabulary, forking the beams' pages, copying pages, moving the
accepted path of a verified tree together, and distillation of a draft from the target's top
logits (loss and gradient).

``run`` computes each operator from elementary torch operations, or with ``own`` by the
calls of paper_2410_05165_amd.paged and .align.  ``exact`` computes it in 64 bits from the
definition.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # One beam level of one user's top-10 list over the item codes of a small fp32 model: latency alone.
        dict(name="select_one_user", op="select", users=1, beams=10, k=10, cols=1024, dtype="fp32", masked=0.75,
             ends=False, log_probs=False, path=4),
        # 32 users of the 7B-shaped target, beams that may end, over the whole vocabulary.
        dict(name="select_vocab", op="select", users=32, beams=10, k=10, cols=33024, dtype="bf16", masked=0.0,
             ends=True, log_probs=False, path=64),
        # 128 users of 50 beams over the whole vocabulary: the widest lists.
        dict(name="select_stress", op="select", users=128, beams=50, k=50, cols=33024, dtype="bf16", masked=0.0,
             ends=False, log_probs=False, path=4),
        # The ten beams of one user behind a prefix of 84 tokens.
        dict(name="fork_one_user", op="fork", users=1, beams=10, held=84, page=16, layers=1),
        # 100 users of ten beams with histories of up to 4,096 tokens.
        dict(name="fork_batch", op="fork", users=100, beams=10, held=4096, page=16, layers=1),
        # The last pages of one user's beams on a two-layer fp32 model, 4 heads of 32.
        dict(name="copy_one_user", op="copy", rows=10, layers=2, kv_heads=4, dh=32, page=16, dtype="fp32"),
        # The last pages of 320 beams, 32 layers of 8 heads of 128.
        dict(name="copy_batch", op="copy", rows=320, layers=32, kv_heads=8, dh=128, page=16, dtype="bf16"),
        # The four accepted nodes of one user's 30 on the two-layer model.
        dict(name="compact_one_user", op="compact", users=1, ctx=80, new=30, path=4, layers=2, kv_heads=4, dh=32,
             page=16, dtype="fp32"),
        # Accepted paths of up to eight nodes of 128 users' trees of 300, 32 layers of 8 heads of 128.
        dict(name="compact_batch", op="compact", users=128, ctx=1024, new=300, path=8, layers=32, kv_heads=8, dh=128,
             page=64, dtype="bf16"),
        # The contexts of 16 users' lists (40 nodes each) over the item codes, ten teacher codes.
        dict(name="distill_items", op="distill", rows=640, cols=1024, tops=10, dtype="fp32", temperature=1.0, rest=False,
             reverse=False),
        # 2,048 positions over the whole vocabulary, 64 teacher logits and the mass of the others.
        dict(name="distill_vocab", op="distill", rows=2048, cols=33024, tops=64, dtype="bf16", temperature=2.0, rest=True,
             reverse=False),
        # 8,192 positions, fp32 logits, the reverse divergence: the largest.
        dict(name="distill_reverse", op="distill", rows=8192, cols=33024, tops=32, dtype="fp32", temperature=1.0, rest=True,
             reverse=True),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    op = rng.choice(["select", "select", "fork", "copy", "compact", "distill", "distill"])
    page = rng.choice([8, 16, 32, 64])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op == "select":
        cols, beams = _spread(rng, 200, 60000), _spread(rng, 1, 64)
        most = 6400 * 33024 * 2 // (cols * beams * (2 if dtype == "bf16" else 4))
        return dict(op=op, users=_spread(rng, 1, max(1, min(128, most))), beams=beams, k=_spread(rng, 1, 128), cols=cols,
                    dtype=dtype, masked=rng.choice([0.0, 0.0, 0.5, 0.97]), ends=rng.random() < 0.4,
                    log_probs=rng.random() < 0.2, path=_spread(rng, 1, 128))
    if op == "fork":
        beams = _spread(rng, 1, 50)
        return dict(op=op, users=_spread(rng, 1, 1000 // beams), beams=beams, held=_spread(rng, 1, 4096), page=max(16, page),
                    layers=1)
    layers, kv, dh = _spread(rng, 1, 32), rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
    if op == "copy":
        most = 320 * 2_097_152 // (layers * 2 * page * kv * dh * (2 if dtype == "bf16" else 4))
        return dict(op=op, rows=_spread(rng, 1, min(1000, most)), layers=layers, kv_heads=kv, dh=dh, page=page, dtype=dtype)
    if op == "compact":
        new = _spread(rng, 2, 300)
        most = 128 * 1324 * 131072 // (layers * 2 * (1024 + new) * kv * dh * (2 if dtype == "bf16" else 4))
        return dict(op=op, users=_spread(rng, 1, min(128, most)), ctx=_spread(rng, 1, 1024), new=new,
                    path=_spread(rng, 1, min(new, 16)), layers=layers, kv_heads=kv, dh=dh, page=page, dtype=dtype)
    cols = _spread(rng, 200, 131072)
    rest = rng.random() < 0.6
    return dict(op=op, rows=_spread(rng, 1, min(8192, 8192 * 33024 // cols)), cols=cols, tops=_spread(rng, 1, 150),
                dtype=dtype, temperature=rng.choice([0.5, 1.0, 1.0, 2.0]), rest=rest, reverse=rest and rng.random() < 0.5)


# ---------------------------------------------------------------- inputs

def _lengths(n, top, low=None):
    """Lengths of up to top, most between a few tokens and all of it: the case's own, whatever the inputs."""
    if n == 1:
        return np.full(1, top, np.int64)
    r = np.random.default_rng([n, top])
    low = max(1, top / 24) if low is None else low
    x = np.minimum(top, np.maximum(1, np.round(np.exp(r.uniform(math.log(low), math.log(top + 0.5), n)))))
    x[0] = top
    return x.astype(np.int64)


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _floats(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV)


def _randn(g, shape, dtype, scale=1.0):
    """Normal values, made piece by piece in the wanted type."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat, piece = out.view(-1), 1 << 26
    for at in range(0, flat.numel(), piece):
        part = flat[at:at + piece]
        part.copy_(torch.randn(part.numel(), generator=g, device=DEV, dtype=torch.float32) * scale)
    return out


def _caches(g, c, pool):
    shape = (c["layers"], pool, c["page"], c["kv_heads"], c["dh"])
    return _randn(g, shape, TYPES[c["dtype"]]), _randn(g, shape, TYPES[c["dtype"]])


def prepare(case, seed):
    r = np.random.default_rng(seed)
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    c = case
    s = dict(case=c)
    if c["op"] == "select":
        U, V = c["users"], c["cols"]
        count = _lengths(U, c["beams"], max(1, c["beams"] * 3 / 4))       # most lists are full
        rows = int(count.sum())
        logits = _randn(g, (rows, V), TYPES[c["dtype"]], 3.0)
        if c["log_probs"]:
            logits.copy_(logits.float() - 9.0)
        if c["masked"] > 0:                                               # columns that a grammar rules out
            for at in range(0, rows, 256):
                piece = logits[at:at + 256]
                piece.masked_fill_(torch.rand(piece.shape, generator=g, device=DEV) < c["masked"], -math.inf)
        held = r.integers(0, c["path"], rows)
        s.update(logits=logits, row_off=_ints(np.concatenate([[0], np.cumsum(count)])), score=_floats(-r.gamma(4.0, 2.0, rows)),
                 done=_ints(r.random(rows) < 0.1) if c["ends"] else None, row_id=_ints(r.permutation(rows)),
                 paths=_ints(r.integers(0, V, (rows, c["path"]))), path_len=_ints(held))
    elif c["op"] == "fork":
        U, K, page = c["users"], c["beams"], c["page"]
        B, length = U * K, _lengths(U, c["held"])
        most = -(-(c["held"] + 8) // page)
        # a user's beams share the pages of the prefix; the last two pages are each beam's own
        need = -(-length // page)
        joint = np.maximum(need - 2, 0)
        alone = need - joint
        pool = int(joint.sum() + K * alone.sum()) + 2 * B + 8
        order = r.permutation(pool).astype(np.int32)
        table, at = np.full((U, K, most), -1, np.int32), 0
        shared = np.zeros(pool, np.int32)
        for u in range(U):
            table[u, :, :joint[u]] = order[at:at + joint[u]]
            shared[order[at:at + joint[u]]] = K - 1
            at += int(joint[u])
            table[u, :, joint[u]:need[u]] = order[at:at + K * alone[u]].reshape(K, alone[u])
            at += int(K * alone[u])
        free = np.full(pool, -1, np.int32)
        free[:pool - at] = order[at:]
        # few beams have most of the children
        src = np.arange(U)[:, None] * K + np.minimum(np.floor(K * r.random((U, K)) ** 2), K - 1)
        s.update(held=_ints(np.repeat(length, K)), keep=_ints(np.repeat(length, K)), src=_ints(src.reshape(-1)),
                 table=_ints(table.reshape(B, most)), free=_ints(free), n_free=_ints([pool - at]), shared=_ints(shared))
    elif c["op"] == "copy":
        n, page = c["rows"], c["page"]
        pool = 2 * n + 4
        order = r.permutation(pool)
        length = r.integers(1, page, n)
        length[r.random(n) < 0.1] = 0                                     # beams that go on in place
        src = np.where(r.random(n) < 0.5, order[0], order[:n]) if n > 1 else order[:n]
        s.update(src=_ints(src), dst=_ints(np.where(length > 0, order[n:2 * n], -1)), length=_ints(length))
        s["k_cache"], s["v_cache"] = _caches(g, c, pool)
    elif c["op"] == "compact":
        U, page, P = c["users"], c["page"], c["path"]
        ctx, new = _lengths(U, c["ctx"]), _lengths(U, c["new"], max(1, c["new"] / 2))
        need = -(-(ctx + new) // page)
        pool = int(need.sum()) + 4
        order, table, at = r.permutation(pool), np.full((U, int(need.max())), -1, np.int32), 0
        path, n_path = np.full((U, P), -1, np.int32), np.minimum(_lengths(U, P), new)
        for u in range(U):
            table[u, :need[u]] = order[at:at + need[u]]
            at += int(need[u])
            path[u, :n_path[u]] = np.sort(r.choice(int(new[u]), int(n_path[u]), replace=False))
        s.update(table=_ints(table), ctx=_ints(ctx), path=_ints(path), n_path=_ints(n_path))
        s["k_cache"], s["v_cache"] = _caches(g, c, pool)
    else:
        n, V, m, T = c["rows"], c["cols"], c["tops"], c["temperature"]
        logits = _randn(g, (n, V), TYPES[c["dtype"]], 2.0)
        step = r.integers(1, max(2, V // m), n)
        index = (r.integers(0, V, n)[:, None] + step[:, None] * np.arange(m)) % V       # distinct columns
        teacher = -np.sort(-r.normal(6.0, 2.5, (n, m)), axis=1)
        index = _ints(index)
        teacher = _floats(teacher)
        # the student has learned part of it
        there = 0.7 * teacher + _randn(g, (n, m), torch.float32, 1.0) + 1.0
        logits.scatter_(1, index.long(), there.to(logits.dtype))
        if m > 2:                                                          # rows with fewer teacher logits
            short = _ints(r.random(n) < 0.05).bool()
            index[short, -(m // 3):] = -1
        part = _floats(r.uniform(0.02, 0.4, n))
        rest = torch.logsumexp(teacher / T, 1) + torch.log(part / (1 - part))
        s.update(logits=logits, index=index, teacher=teacher.to(logits.dtype), rest=rest if c["rest"] else None,
                 weight=_floats(r.uniform(0.2, 1.0, n) / n), grad_loss=_floats(r.uniform(0.5, 1.5, n)))
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return _RUN[s["case"]["op"]](s)


def _top_keys(x, k):
    """The k largest of each row of x, fp32 without NaN, largest first, and their columns: equal ones from the lowest."""
    bits = x.contiguous().view(torch.int32).long()
    bits = torch.where(x == 0, 0, bits)                                     # -0 and 0 are equal
    order = torch.where(bits < 0, ~bits & 0xffffffff, bits | 0x80000000)   # ascending with x, 32 bits
    col = torch.arange(x.shape[1], device=DEV)
    key = ((order - 0x80000000) << 32) | (0xffffffff - col)
    at = 0xffffffff - (torch.topk(key, k, dim=1).values & 0xffffffff)
    return torch.gather(x, 1, at), at


def _run_select(s):
    c = s["case"]
    if own:
        from paper_2410_05165_amd.paged import atspeed_beam_select
        b = atspeed_beam_select(s["logits"], s["row_off"], c["k"], score=s["score"], done=s["done"], token_base=0,
                                log_probs=c["log_probs"], row_id=s["row_id"], paths=s["paths"], path_len=s["path_len"])
        return dict(count=b.count, parent=b.parent, token=b.token, score=b.score, paths=b.paths, path_len=b.path_len)
    x = s["logits"].float()
    rows, V = x.shape
    U, R, k, P = c["users"], c["beams"], c["k"], c["path"]
    row_off = s["row_off"].long()
    n = min(k, V)
    value, col = _top_keys(x, n)                                            # [rows, n]
    if c["log_probs"]:
        lse = torch.zeros(rows, dtype=torch.float64, device=DEV)
    else:                                                                   # 64 bits: scores of different beams rank together
        top = x.amax(1).double()
        lse = top + torch.log(torch.exp(x.double() - top[:, None]).sum(1))
    cand = (s["score"].double() - lse)[:, None] + value.double()
    cand = torch.where(value > -math.inf, cand, -math.inf)
    if s["done"] is not None:
        ended = s["done"].bool()
        cand[ended] = -math.inf
        cand[ended, 0] = s["score"].double()[ended]
        col = torch.where(ended[:, None], -1, col)
    # a request's candidates, its rows in order
    user = torch.searchsorted(row_off[1:].contiguous(), torch.arange(rows, device=DEV), right=True)
    i = torch.arange(rows, device=DEV) - row_off[user]
    pool = torch.full((U, R, n), -math.inf, dtype=torch.float64, device=DEV)
    pool[user, i] = cand
    best, at = torch.sort(pool.view(U, R * n), dim=1, descending=True, stable=True)
    if R * n < k:
        best = torch.cat([best, torch.full((U, k - R * n), -math.inf, dtype=torch.float64, device=DEV)], 1)
        at = torch.cat([at, torch.zeros((U, k - R * n), dtype=torch.long, device=DEV)], 1)
    best, at = best[:, :k], at[:, :k]
    live = best > -math.inf
    row = torch.where(live, row_off[:-1, None] + at // n, 0)
    who = s["row_id"].long()[row]
    token = torch.where(live, col[row, at % n], -1)
    held = s["path_len"].long()[who]
    paths = torch.where(torch.arange(P, device=DEV) < held[:, :, None], s["paths"].long()[who], -1)
    grows = live & (token >= 0) & (held < P)
    spot = held.clamp(max=P - 1)[:, :, None]
    paths = paths.scatter(2, spot, torch.where(grows[:, :, None], token[:, :, None], torch.gather(paths, 2, spot)))
    return dict(count=live.sum(1).int(), parent=torch.where(live, who, -1).int(), token=token.int(),
                score=torch.where(live, best, -math.inf).float(), paths=torch.where(live[:, :, None], paths, -1).int(),
                path_len=torch.where(live, held + grows.long(), 0).int())


def _run_fork(s):
    if own:
        from paper_2410_05165_amd.paged import atspeed_page_fork
        f = atspeed_page_fork(s["held"], s["keep"], s["table"], s["free"], s["n_free"], s["shared"], s["case"]["page"],
                              src=s["src"])
        return dict(table=s["table"], free=s["free"], n_free=s["n_free"], shared=s["shared"], length=f.length,
                    refused=f.refused, copy_src=f.copy_src, copy_dst=f.copy_dst, copy_len=f.copy_len)
    page = s["case"]["page"]
    held, keep, src, table, shared = (s[k].long() for k in ("held", "keep", "src", "table", "shared"))
    (B, most), pool = table.shape, s["free"].numel()
    row = torch.arange(B, device=DEV)
    held = torch.where((held < 0) | (held > most * page), 0, held)
    bad = (src < -1) | (src >= B)
    bad = bad | ((src != -1) & ((keep < 0) | (keep > held[src.clamp(0, B - 1)])))
    frm = torch.where(bad, row, src)
    kept = torch.where(bad, held, torch.where(frm < 0, 0, keep))
    frm = frm.clamp(min=0)
    full, over = kept // page, kept % page
    col = torch.arange(most, device=DEV)
    sound = (table >= 0) & (table < pool)
    count = lambda where, pages: torch.zeros(pool, dtype=torch.long, device=DEV).scatter_add_(  # noqa: E731
        0, torch.where(where, pages, 0).view(-1), where.long().view(-1))
    olds = (col < ((held + page - 1) // page)[:, None]) & sound
    news = (col < full[:, None]) & sound[frm]
    was, stays = count(olds, table), count(news, table[frm])
    tail = table[frm, full.clamp(max=most - 1)]
    wants = (over > 0) & (tail >= 0) & (tail < pool)
    spot = tail.clamp(0, pool - 1)
    first = torch.full((pool,), B, device=DEV).scatter_reduce_(0, spot, torch.where(wants, row, B), "amin")
    others = shared - was                                                   # holders that are no rows, less one
    takes = wants & (stays[spot] == 0) & (others[spot] < 0) & (first[spot] == row)
    left = others + stays + count(takes, spot)
    gone = (was > 0) & (left < 0)
    # released pages are pushed in ascending order, then the wanted ones popped in the rows' order
    F = s["n_free"].long()
    place = F + torch.cumsum(gone.long(), 0) - 1
    stack = s["free"].long().clone()
    every = torch.arange(pool, device=DEV)
    stack = torch.cat([stack, stack[:1]]).scatter(0, torch.where(gone, place, pool).clamp(max=pool), every)[:pool]
    have = (F + gone.sum()).clamp(max=pool)
    copies = wants & ~takes
    rank = torch.cumsum(copies.long(), 0)
    short = copies & (rank > have)
    copies = copies & ~short
    fresh = stack[(have - rank).clamp(0, pool - 1)]
    n_free = have - copies.sum()
    new = torch.where(col < full[:, None], table[frm], table)
    at_tail = (col == full[:, None]) & (over > 0)[:, None] & ~short[:, None]
    new = torch.where(at_tail, torch.where(copies, fresh, tail)[:, None], new)
    s["free"].copy_(torch.where(every < n_free, stack, s["free"].long()))
    s["table"].copy_(new)
    s["shared"].copy_(torch.where(was > 0, left.clamp(min=0), shared))
    s["n_free"].copy_(n_free)
    return dict(table=s["table"], free=s["free"], n_free=s["n_free"], shared=s["shared"],
                length=torch.where(short, full * page, kept).int(), refused=torch.where(bad, 2, short.long()).int(),
                copy_src=torch.where(copies, tail, -1).int(), copy_dst=torch.where(copies, fresh, -1).int(),
                copy_len=torch.where(copies, over, 0).int())


def _move(s, src, dst):
    """Token slots src to dst, in every layer."""
    for name in ("k_cache", "v_cache"):
        cache = s[name]
        slots = cache.view(cache.shape[0], -1, *cache.shape[3:])
        slots[:, dst] = slots[:, src]
    return dict(k_cache=s["k_cache"], v_cache=s["v_cache"])


def _run_copy(s):
    if own:
        from paper_2410_05165_amd.paged import atspeed_page_copy
        atspeed_page_copy(s["k_cache"], s["v_cache"], s["src"], s["dst"], s["length"])
        return dict(k_cache=s["k_cache"], v_cache=s["v_cache"])
    page = s["case"]["page"]
    t = torch.arange(page, device=DEV)
    live = (t < s["length"][:, None]) & (s["dst"] >= 0)[:, None]
    return _move(s, (s["src"].long()[:, None] * page + t)[live], (s["dst"].long()[:, None] * page + t)[live])


def _run_compact(s):
    if own:
        from paper_2410_05165_amd.paged import atspeed_kv_compact
        atspeed_kv_compact(s["k_cache"], s["v_cache"], s["table"], s["ctx"], s["path"], s["n_path"])
        return dict(k_cache=s["k_cache"], v_cache=s["v_cache"])
    page, ctx = s["case"]["page"], s["ctx"].long()
    i = torch.arange(s["path"].shape[1], device=DEV)
    live = i < s["n_path"][:, None]
    slot = lambda p: torch.gather(s["table"].long(), 1, p // page) * page + p % page  # noqa: E731
    frm = slot(ctx[:, None] + torch.where(live, s["path"].long(), 0))
    to = slot(ctx[:, None] + torch.where(live, i, 0))
    return _move(s, frm[live], to[live])


def _run_distill(s):
    c = s["case"]
    T, rest, weight = c["temperature"], s["rest"], s["weight"]
    if own:
        from paper_2410_05165_amd.align import atspeed_distill_grad, atspeed_distill_loss
        loss, saved = atspeed_distill_loss(s["logits"], s["teacher"], s["index"], tail=rest, weight=weight, temperature=T,
                                           reverse=c["reverse"])
        return dict(loss=loss, grad=atspeed_distill_grad(s["logits"], s["index"], saved, s["grad_loss"], temperature=T))
    index = s["index"].long()
    there = index >= 0
    index = index.clamp(min=0)
    # the teacher's buckets: its logits, and the rest
    t = torch.where(there, s["teacher"].float() / T, -math.inf)
    t = torch.cat([t, rest[:, None] if rest is not None else torch.full_like(t[:, :1], -math.inf)], 1).double()
    t = t - t.amax(1, keepdim=True)
    log_p = t - torch.log(torch.exp(t).sum(1, keepdim=True))
    p = torch.exp(log_p)
    z = s["logits"].float() / T
    e = torch.exp(z - z.amax(1, keepdim=True))
    top = torch.where(there, torch.gather(e, 1, index), 0.0)
    outside = torch.ones_like(e).scatter_reduce_(1, index, torch.where(there, 0.0, 1.0), "amin")
    others = (e * outside).sum(1).double()
    total = others + top.double().sum(1)
    q = torch.cat([top.double(), others[:, None]], 1) / total[:, None]      # the student's buckets
    zt = torch.gather(z, 1, index).double() - z.amax(1, keepdim=True).double()
    log_q = torch.cat([zt, torch.log(others)[:, None]], 1) - torch.log(total)[:, None]
    if c["reverse"]:
        far = torch.where(q > 0, log_q - log_p, 0.0)
        loss = (q * far).sum(1)
        at_top, else_ = q[:, :-1] * (far[:, :-1] - loss[:, None]), far[:, -1] - loss
    else:
        loss = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
        at_top, else_ = q[:, :-1] - p[:, :-1], 1.0 - p[:, -1] / q[:, -1]
    step = s["grad_loss"] * weight * T
    grad = e
    grad *= (step * else_.float() / total.float())[:, None]
    spot, at_top = torch.where(there, index, index[:, :1]), torch.where(there, at_top, at_top[:, :1])
    grad.scatter_(1, spot, step[:, None] * at_top.float())
    return dict(loss=(weight * T * T * loss).float(), grad=grad.to(s["logits"].dtype))


_RUN = dict(select=_run_select, fork=_run_fork, copy=_run_copy, compact=_run_compact, distill=_run_distill)


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    c = case
    if c["op"] == "fork":
        return None                                    # whole numbers
    s = prepare(case, seed)
    if c["op"] == "select":
        off, k, V = s["row_off"].tolist(), c["k"], c["cols"]
        score = torch.full((c["users"], k), -math.inf, dtype=torch.float64, device=DEV)
        for u in range(c["users"]):
            x = s["logits"][off[u]:off[u + 1]].double()
            if not c["log_probs"]:
                x = torch.log_softmax(x, 1)
            x = torch.nan_to_num(x, nan=-math.inf, neginf=-math.inf) + s["score"][off[u]:off[u + 1], None].double()
            if s["done"] is not None:
                for r in range(off[u], off[u + 1]):
                    if int(s["done"][r]):
                        x[r - off[u]] = -math.inf
                        x[r - off[u], 0] = s["score"][r].double()
            best = torch.sort(x.reshape(-1), descending=True).values[:k]
            score[u, :best.numel()] = best
        return dict(count=None, parent=None, token=None, score=score, paths=None, path_len=None)
    if c["op"] in ("copy", "compact"):
        k, v = s["k_cache"].double(), s["v_cache"].double()
        page = c["page"]
        if c["op"] == "copy":
            for a, b, n in zip(s["src"].tolist(), s["dst"].tolist(), s["length"].tolist()):
                if b >= 0:
                    for x in (k, v):
                        x[:, b, :n] = x[:, a, :n].clone()
        else:
            table = s["table"].tolist()
            for u, (ctx, n) in enumerate(zip(s["ctx"].tolist(), s["n_path"].tolist())):
                for i, node in enumerate(s["path"][u, :n].tolist()):        # in order: no node lies below its place
                    a, b = ctx + node, ctx + i
                    for x in (k, v):
                        x[:, table[u][b // page], b % page] = x[:, table[u][a // page], a % page].clone()
        return dict(k_cache=k, v_cache=v)
    T, V = c["temperature"], c["cols"]
    n = c["rows"]
    loss = torch.empty(n, dtype=torch.float64, device=DEV)
    grad = torch.empty((n, V), dtype=torch.float64, device=DEV)
    piece = max(1, (1 << 26) // V)
    for at in range(0, n, piece):
        z = (s["logits"][at:at + piece].double() / T).requires_grad_()
        index, teacher = s["index"][at:at + piece].long(), s["teacher"][at:at + piece].double() / T
        teacher = teacher.masked_fill(index < 0, -math.inf)
        if s["rest"] is not None:
            teacher = torch.cat([teacher, s["rest"][at:at + piece, None].double()], 1)
        log_p = torch.log_softmax(teacher, 1)
        log_q = torch.log_softmax(z, 1)
        tops = torch.gather(log_q, 1, index.clamp(min=0)).masked_fill(index < 0, 0.0)
        if s["rest"] is not None:
            mine = torch.zeros((z.shape[0], V + 1), dtype=torch.bool, device=DEV)
            mine.scatter_(1, torch.where(index >= 0, index, V), True)
            tops = torch.cat([tops, torch.logsumexp(log_q.masked_fill(mine[:, :V], -math.inf), 1)[:, None]], 1)
        live = log_p > -math.inf
        log_p = torch.where(live, log_p, 0.0)
        if c["reverse"]:
            each = torch.where(live, torch.exp(tops) * (tops - log_p), 0.0).sum(1)
        else:
            each = torch.where(live, torch.exp(log_p) * (log_p - tops), 0.0).sum(1)
        each = each * s["weight"][at:at + piece].double() * T * T
        # with respect to the logits, which are T times z
        grad[at:at + piece] = torch.autograd.grad((each * s["grad_loss"][at:at + piece].double()).sum(), z)[0] / T
        loss[at:at + piece] = each.detach()
    return dict(loss=loss, grad=grad)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    es = 2 if c.get("dtype") == "bf16" else 4
    if c["op"] == "select":
        rows = int(_lengths(c["users"], c["beams"], max(1, c["beams"] * 3 / 4)).sum())
        # one exponential and a comparison an element
        return dict(bytes=rows * (c["cols"] * es + 12) + c["users"] * c["k"] * (16 + 8 * c["path"]), flops=3.0 * rows * c["cols"])
    if c["op"] == "fork":
        pages = int(-(-_lengths(c["users"], c["held"]) // c["page"]).sum()) * c["beams"]
        # the entries, read and written, the lengths, and the count of each page
        return dict(bytes=8 * pages + 32 * c["users"] * c["beams"] + 8 * pages // c["beams"], flops=pages)
    if c["op"] == "copy":
        token = 2 * c["layers"] * c["kv_heads"] * c["dh"] * es
        return dict(bytes=2 * 0.9 * c["rows"] * c["page"] / 2 * token, flops=0)
    if c["op"] == "compact":
        token = 2 * c["layers"] * c["kv_heads"] * c["dh"] * es
        moved = int(np.minimum(_lengths(c["users"], c["path"]), _lengths(c["users"], c["new"], max(1, c["new"] / 2))).sum())
        return dict(bytes=2 * moved * token, flops=0)
    n, V, m = c["rows"], c["cols"], c["tops"]
    # the logits once for the loss and once for the gradient, which is written once
    return dict(bytes=3 * n * V * es + n * m * (es + 4) + 16 * n, flops=8.0 * n * V)

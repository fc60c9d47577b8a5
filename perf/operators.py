"""Measured cases of the operators that verify drafted trees on a caller's own target:
the step plan over a paged cache, the append of new keys and values, tree attention over
the pages, and the rules on the logits (penalties, biases, grammar masks).

``run`` computes each operator from elementary torch operations, or with ``own`` by the
calls of paper_2410_05165_amd.paged.  ``exact`` computes it in 64 bits from the definition.
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
        # One user's drafted tree over a prefix of 80 tokens (fp32, 30 nodes): latency alone.
        dict(name="plan_one_user", op="plan", users=1, held=80, new=30, levels=3, page=16, tree=True),
        # A full serving batch with histories of up to 4,096 tokens, trees of up to 110 nodes.
        dict(name="plan_batch", op="plan", users=1024, held=4096, new=110, levels=4, page=16, tree=True),
        # The tree rows of 32 users (60 nodes each) of a 7B-shaped target, 32 heads of 128.
        dict(name="append_verify", op="append", users=32, new=60, heads=32, kv_heads=32, dh=128, page=64, dtype="bf16"),
        # Prefill chunks of 32 users with grouped heads, out of the rows of a fused projection.
        dict(name="append_prefill", op="append", users=32, new=1024, heads=32, kv_heads=8, dh=128, page=16, dtype="bf16"),
        # One user's tree on a two-layer fp32 model: 4 heads of 32 over 80 tokens.
        dict(name="attn_one_user", op="attention", users=1, ctx=80, new=30, levels=3, heads=4, kv_heads=4, dh=32,
             page=16, dtype="fp32", tree=True, ragged=False),
        # The verify of 32 users, 60 nodes each, over the prompt and history of 144 tokens.
        dict(name="attn_verify", op="attention", users=32, ctx=144, new=60, levels=3, heads=32, kv_heads=32, dh=128,
             page=64, dtype="bf16", tree=True, ragged=False),
        # 128 users with histories around 1,024 tokens and 300 drafted nodes: the largest.
        dict(name="attn_stress", op="attention", users=128, ctx=1024, new=300, levels=3, heads=32, kv_heads=32, dh=128,
             page=64, dtype="bf16", tree=True, ragged=False),
        # Single tokens of 64 requests of very different lengths, grouped heads, small pages.
        dict(name="attn_decode", op="attention", users=64, ctx=8192, new=1, levels=1, heads=32, kv_heads=8, dh=128,
             page=16, dtype="bf16", tree=False, ragged=True),
        # Trees of four users behind long contexts.
        dict(name="attn_long", op="attention", users=4, ctx=65536, new=32, levels=3, heads=32, kv_heads=8, dh=128,
             page=32, dtype="bf16", tree=True, ragged=True),
        # Prompt chunks of up to 1,024 tokens over contexts of up to 1,024, causal.
        dict(name="attn_prefill", op="attention", users=16, ctx=1024, new=1024, levels=1, heads=32, kv_heads=8, dh=128,
             page=16, dtype="bf16", tree=False, ragged=True),
        # Item logits of the verified trees of 32 users (61 rows of 4 x 256 codes), short histories.
        dict(name="rules_items", op="rules", users=32, new=61, levels=4, cols=1024, hist=80, dtype="fp32", tree=True,
             states=512),
        # Whole-vocabulary logits of single tokens, long histories.
        dict(name="rules_vocab", op="rules", users=128, new=1, levels=1, cols=33024, hist=2048, dtype="bf16", tree=False,
             states=16),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    op = rng.choice(["plan", "append", "attention", "attention", "rules"])
    page = rng.choice([8, 16, 32, 64, 128])
    if op == "plan":
        return dict(op=op, users=_spread(rng, 1, 1024), held=_spread(rng, 1, 8192), new=_spread(rng, 1, 128),
                    levels=rng.randint(1, 6), page=page, tree=rng.random() < 0.7)
    if op == "append":
        kv = rng.choice([1, 2, 4, 8, 12, 16, 32])
        return dict(op=op, users=_spread(rng, 1, 64), new=_spread(rng, 1, 500), heads=kv * rng.choice([1, 2, 4]),
                    kv_heads=kv, dh=rng.choice([64, 128]), page=page, dtype=rng.choice(["bf16", "bf16", "fp32"]))
    if op == "rules":
        tree = rng.random() < 0.5
        return dict(op=op, users=_spread(rng, 1, 64), new=_spread(rng, 2, 90) if tree else 1, levels=rng.randint(1, 6),
                    cols=_spread(rng, 200, 1024) if tree else _spread(rng, 1000, 60000), hist=_spread(rng, 1, 2048),
                    dtype=rng.choice(["fp32", "bf16"]), tree=tree, states=_spread(rng, 1, 300))
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    tree = rng.random() < 0.6
    kv = rng.choice([1, 2, 4, 8, 12])
    new = 1 if not tree and rng.random() < 0.5 else _spread(rng, 2, 300 if tree else 700)
    ctx = _spread(rng, 1, 16384 if new < 40 else 2048)
    heads = kv * rng.choice([1, 2, 3, 4, 8])
    most = min(64, 120000 // (ctx + new), 1_200_000_000 // (new * (ctx + new) * heads))   # no more than the largest above
    return dict(op=op, users=_spread(rng, 1, max(1, most)), ctx=ctx, new=new, levels=rng.randint(1, 6), heads=heads,
                kv_heads=kv, dh=rng.choice([64, 128] if dtype == "bf16" else [32, 64, 128]), page=page, dtype=dtype,
                tree=tree, ragged=rng.random() < 0.7)


# ---------------------------------------------------------------- inputs

def _lengths(n, top, ragged=True):
    """Request lengths of up to top, between a few tokens and all of it: the case's own, whatever the inputs."""
    if not ragged or n == 1:
        return np.full(n, top, np.int64)
    r = np.random.default_rng([n, top])
    x = np.minimum(top, np.maximum(1, np.round(np.exp(r.uniform(math.log(max(1, top / 24)), math.log(top + 0.5), n)))))
    x[0] = top
    return x.astype(np.int64)


def _tree(r, n, levels):
    """A level-ordered tree of n nodes: each level about the same width, parents among the level above."""
    sizes = [len(p) for p in np.array_split(np.arange(n), max(1, min(levels, n)))]
    parent, above, at = np.empty(n, np.int32), None, 0
    for width in sizes:
        parent[at:at + width] = -1 if above is None else above[0] + r.integers(0, above[1], width)
        above, at = (at, width), at + width
    return parent


def _forest(r, users, new, levels, top):
    parent = np.full((users, top), -1, np.int32)
    for u in range(users):
        parent[u, :new[u]] = _tree(r, int(new[u]), levels)
    return parent


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _words(top):
    return (top + 63) // 64


def _mask_of(parent, new):
    """Ancestor-or-self bits of every row, rows packed by request: [rows, words] int64."""
    users, top = parent.shape
    seen = np.zeros((users, top, _words(top) * 64), bool)
    who = np.arange(users)
    for i in range(top):
        p = parent[:, i]
        seen[:, i] = seen[who, np.maximum(p, 0)] & (p >= 0)[:, None]
        seen[:, i, i] = True
    live = np.arange(top)[None, :] < new[:, None]
    bits = np.packbits(seen[live], axis=-1, bitorder="little")
    return torch.from_numpy(bits.view(np.int64).copy()).to(DEV)


def _randn(g, shape, dtype, scale=1.0):
    """Normal values, made piece by piece in the wanted type."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat, piece = out.view(-1), 1 << 26
    for at in range(0, flat.numel(), piece):
        part = flat[at:at + piece]
        part.copy_(torch.randn(part.numel(), generator=g, device=DEV, dtype=torch.float32) * scale)
    return out


def _pages(r, need, most, pool):
    """Block tables [users, most] over a shuffled pool, and the pages that are free."""
    order = r.permutation(pool).astype(np.int32)
    table = np.full((len(need), most), -1, np.int32)
    table[np.arange(most)[None, :] < need[:, None]] = order[:int(need.sum())]
    return table, order[int(need.sum()):]


def prepare(case, seed):
    r = np.random.default_rng(seed)
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    c, U = case, case["users"]
    s = dict(case=c)
    if c["op"] == "plan":
        page, top = c["page"], c["new"]
        held = _lengths(U, c["held"])
        # most requests keep what they hold, some drop drafted tokens, some have ended, some are new
        kind = r.random(U)
        keep = np.where(kind < 0.6, held, np.where(kind < 0.9, np.maximum(0, held - r.integers(0, top + 1, U)), 0))
        held = np.where(kind > 0.97, 0, held)
        keep = np.minimum(keep, held)
        new = np.where((kind >= 0.9) & (kind <= 0.95), 0, _lengths(U, top))
        before = -(-held // page)
        most = -(-(c["held"] + top) // page)
        pool = U * most + 8
        table, rest = _pages(r, before, most, pool)
        free = np.full(pool, -1, np.int32)
        free[:len(rest)] = rest
        s.update(held=_ints(held), keep=_ints(keep), add=_ints(new), table=_ints(table), free=_ints(free),
                 n_free=_ints([len(rest)]), page=page, max_rows=U * top,
                 parent=_ints(_forest(r, U, new, c["levels"], top)) if c["tree"] else None)
    elif c["op"] == "append":
        page, H, K, dh, dtype = c["page"], c["heads"], c["kv_heads"], c["dh"], TYPES[c["dtype"]]
        new = _lengths(U, c["new"])
        keep = r.integers(0, 4 * page + 1, U)
        most = 4 + -(-c["new"] // page)
        pool = U * most
        table, _ = _pages(r, -(-(keep + new) // page), most, pool)
        row_off = np.concatenate([[0], np.cumsum(new)])
        user = np.repeat(np.arange(U), new)
        pos = keep[user] + np.arange(row_off[-1]) - row_off[user]
        qkv = _randn(g, (int(row_off[-1]), (H + 2 * K) * dh), dtype)
        s.update(k=qkv[:, H * dh:(H + K) * dh].view(-1, K, dh), v=qkv[:, (H + K) * dh:].view(-1, K, dh),
                 k_cache=_randn(g, (pool, page, K, dh), dtype), v_cache=_randn(g, (pool, page, K, dh), dtype),
                 slot=_ints(table[user, pos // page] * page + pos % page))
    elif c["op"] == "attention":
        page, H, K, dh, dtype = c["page"], c["heads"], c["kv_heads"], c["dh"], TYPES[c["dtype"]]
        ctx, new = _lengths(U, c["ctx"], c["ragged"]), _lengths(U, c["new"], c["ragged"])
        need = -(-(ctx + new) // page)
        pool = int(need.sum()) * 17 // 16 + 4
        table, _ = _pages(r, need, int(need.max()), pool)
        rows = int(new.sum())
        # scores with a spread of about two, as trained heads have
        s.update(q=_randn(g, (rows, H, dh), dtype, 2.0), k_cache=_randn(g, (pool, page, K, dh), dtype),
                 v_cache=_randn(g, (pool, page, K, dh), dtype), table=_ints(table), ctx=_ints(ctx),
                 row_off=_ints(np.concatenate([[0], np.cumsum(new)])),
                 mask=_mask_of(_forest(r, U, new, c["levels"], c["new"]), new) if c["tree"] else None)
    else:
        V = c["cols"]
        new = _lengths(U, c["new"], c["new"] > 1)
        rows, base = int(new.sum()), 32000
        hist = np.minimum(V - 1, np.floor(V * r.random((U, c["hist"])) ** 3)).astype(np.int64) + base
        hist[r.random(hist.shape) < 0.05] = 7                       # tokens outside the columns
        row_off = np.concatenate([[0], np.cumsum(new)])
        words = (V + 31) // 32
        allowed = torch.randint(-2**31, 2**31, (c["states"], words), generator=g, device=DEV, dtype=torch.int64)
        tree = c["tree"]
        logits = _randn(g, (rows, V), TYPES[c["dtype"]], 3.0)
        s.update(logits=logits, row_off=_ints(row_off), history=_ints(hist), hist_len=_ints(_lengths(U, c["hist"])),
                 base=base, repetition=torch.from_numpy(r.uniform(1.0, 1.5, U).astype(np.float32)).to(DEV),
                 frequency=torch.from_numpy(r.uniform(0.0, 0.5, U).astype(np.float32)).to(DEV),
                 presence=torch.from_numpy(r.uniform(0.0, 0.5, U).astype(np.float32)).to(DEV),
                 temperature=torch.from_numpy(r.uniform(0.5, 1.5, U).astype(np.float32)).to(DEV),
                 bias=_randn(g, (3, V), torch.float32, 0.5), bias_index=_ints(r.integers(-1, 3, U)),
                 allowed=allowed.to(torch.int32), state=_ints(r.integers(-1, c["states"], rows)),
                 mask=_mask_of(_forest(r, U, new, c["levels"], c["new"]), new) if tree else None,
                 node_token=_ints(base + r.integers(0, V, (U, c["new"]))) if tree else None)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return _RUN[s["case"]["op"]](s)


def _run_plan(s):
    if own:
        from paper_2410_05165_amd.paged import atspeed_page_plan
        p = atspeed_page_plan(s["held"], s["keep"], s["add"], s["table"], s["free"], s["n_free"], s["page"],
                              s["max_rows"], parent=s["parent"])
        return dict(table=s["table"], free=s["free"], n_free=p.n_free, length=p.length, ctx=p.ctx, refused=p.refused,
                    row_off=p.row_off, row_user=p.row_user, row_pos=p.row_pos, slot=p.slot, tree_slot=p.tree_slot,
                    mask=p.mask)
    held, keep, add, table, free = (s[k].long() for k in ("held", "keep", "add", "table", "free"))
    page, R, (U, most), pool = s["page"], s["max_rows"], table.shape, s["free"].numel()
    top = s["parent"].shape[1] if s["parent"] is not None else R
    F = s["n_free"].long()
    before, after = (held + page - 1) // page, (keep + add + page - 1) // page
    row_off = torch.zeros(U + 1, dtype=torch.long, device=DEV)
    row_off[1:] = torch.cumsum(add, 0)
    bad = (held < 0) | (keep < 0) | (keep > held) | (add < 0) | (before > most) | (after > most) | (add > top)
    bad = bad | (row_off[1:] > R)
    gone = torch.where(bad, 0, (before - after).clamp(min=0))
    want = torch.where(bad, 0, (after - before).clamp(min=0))
    have = F + gone.sum()
    short = (want > 0) & (torch.cumsum(want, 0) > have)
    take = torch.where(short, 0, want)
    ok = ~bad & ~short
    # the stack of free pages: what was free, then the released pages in request order; taken from its top
    g_end, t_end = torch.cumsum(gone, 0), torch.cumsum(take, 0)
    every = torch.arange(pool, device=DEV)
    j = (every - F).clamp(min=0)
    giver = torch.searchsorted(g_end, j, right=True).clamp(max=U - 1)
    at = (after[giver] + j - (g_end - gone)[giver]).clamp(0, most - 1)
    stack = torch.where((every >= F) & (j < g_end[-1]), table[giver, at], free)
    n_free = have - t_end[-1]
    free = torch.where(every < n_free, stack, free)
    col = torch.arange(most, device=DEV)[None, :]
    t = (t_end - take)[:, None] + col - before[:, None]
    fresh = (col >= before[:, None]) & (col < after[:, None]) & ok[:, None]
    table = torch.where(fresh, stack[(have - 1 - t).clamp(0, pool - 1)], table)
    row = torch.arange(R, device=DEV)
    user = torch.searchsorted(row_off[1:].contiguous(), row, right=True)
    live = row < row_off[-1]
    user = torch.where(live, user, 0)
    i = row - row_off[user]
    p = keep[user] + i
    put = live & ok[user]
    slot = table[user, (p // page).clamp(max=most - 1)] * page + p % page
    out = dict(table=table.int(), free=free.int(), n_free=n_free.int(), length=torch.where(ok, keep + add, held).int(),
               ctx=torch.where(ok, keep, -1).int(), refused=torch.where(bad, 2, torch.where(short, 1, 0)).int(),
               row_off=row_off.int(), row_user=torch.where(live, user, -1).int())
    if s["parent"] is None:
        tree_slot, mask, place = torch.where(live, i, -1), None, p
    else:
        W = _words(top)
        parent = s["parent"].long()
        node = torch.arange(top, device=DEV)
        anc = torch.zeros((U, top, W * 64), dtype=torch.bool, device=DEV)
        anc[:, node, node] = True
        jump, who = parent, torch.arange(U, device=DEV)[:, None]
        for _ in range(max(1, (top - 1).bit_length())):       # doubling: twice the ancestors each time
            anc = anc | (anc[who, jump.clamp(min=0)] & (jump >= 0)[:, :, None])
            jump = torch.where(jump >= 0, torch.gather(jump, 1, jump.clamp(min=0)), -1)
        mine = anc[user, i.clamp(0, top - 1)] & put[:, None]
        place = keep[user] + mine.sum(-1) - 1
        weight = torch.ones(64, dtype=torch.long, device=DEV) << torch.arange(64, device=DEV)
        mask = (mine.view(R, W, 64).long() * weight).sum(-1)
        tree_slot = torch.where(live, user * top + i, -1)
    out.update(row_pos=torch.where(put, place, -1).int(), slot=torch.where(put, slot, -1).int(),
               tree_slot=tree_slot.int(), mask=mask)
    return out


def _run_append(s):
    if own:
        from paper_2410_05165_amd.paged import atspeed_kv_append
        atspeed_kv_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slot"])
    else:
        slot = s["slot"].long()
        s["k_cache"].view(-1, *s["k"].shape[1:])[slot] = s["k"]
        s["v_cache"].view(-1, *s["v"].shape[1:])[slot] = s["v"]
    return dict(k_cache=s["k_cache"], v_cache=s["v_cache"])


def _visible(mask, rows, pos, ctx, at, live):
    """Which keys [.., S] at positions pos the rows [U, R] see: the context, and their own path or chain."""
    new = pos[None, None, :] - ctx[:, None, None]
    if mask is None:
        return (new <= at[None, :, None]) & live[:, :, None]
    words = mask[rows]                                                   # [U, R, W]
    bit = new.clamp(0, 64 * mask.shape[1] - 1).expand(rows.shape[0], rows.shape[1], -1)
    word = torch.gather(words, 2, bit // 64)
    set_ = ((word >> (bit % 64)) & 1).bool() & (new < 64 * mask.shape[1])
    return ((new < 0) | set_) & live[:, :, None]


def _run_attention(s):
    c = s["case"]
    H, K, dh, page = c["heads"], c["kv_heads"], c["dh"], c["page"]
    if own:
        from paper_2410_05165_amd.paged import atspeed_tree_attention
        out, lse = atspeed_tree_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["row_off"], s["ctx"],
                                          max_ctx=c["ctx"], max_new=c["new"], mask=s["mask"], return_lse=True)
        return dict(out=out, lse=lse)
    ctx, row_off, q = s["ctx"].long(), s["row_off"].long(), s["q"]
    U, R, S, G = c["users"], c["new"], c["ctx"] + c["new"], H // K
    count = row_off[1:] - row_off[:-1]
    at = torch.arange(R, device=DEV)
    live = at[None, :] < count[:, None]
    rows = torch.where(live, row_off[:-1, None] + at[None, :], 0)
    pos = torch.arange(S, device=DEV)
    slot = s["table"].long()[:, (pos // page).clamp(max=s["table"].shape[1] - 1)].clamp(min=0) * page + pos % page
    held = pos[None, :] < (ctx + count)[:, None]
    keys = s["k_cache"].view(-1, K, dh)[slot].permute(0, 2, 3, 1).float().contiguous()        # [U, K, dh, S]
    queries = q[rows].view(U, R, K, G, dh).permute(0, 2, 1, 3, 4).float().contiguous().view(U, K, R * G, dh)
    score = torch.matmul(queries, keys).view(U, K, R, G, S)
    del keys
    score *= 1.0 / math.sqrt(dh)
    see = (_visible(s["mask"], rows, pos, ctx, at, live) & held[:, None, :])[:, None, :, None, :]
    score.masked_fill_(~see, -math.inf)
    top = score.amax(-1, keepdim=True)
    score -= torch.where(top == -math.inf, 0.0, top)
    score.exp_()
    total = score.sum(-1, keepdim=True)
    values = s["v_cache"].view(-1, K, dh)[slot].permute(0, 2, 1, 3).float().contiguous()      # [U, K, S, dh]
    o = torch.matmul(score.view(U, K, R * G, S), values).view(U, K, R, G, dh)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(U, R, H, dh)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3).reshape(U, R, H)
    n = q.shape[0]
    user = torch.searchsorted(row_off[1:].contiguous(), torch.arange(n, device=DEV), right=True)
    i = torch.arange(n, device=DEV) - row_off[user]
    return dict(out=o[user, i].to(q.dtype), lse=lse[user, i])


def _run_rules(s):
    if own:
        from paper_2410_05165_amd.paged import atspeed_logit_rules
        return atspeed_logit_rules(s["logits"], s["row_off"], token_base=s["base"], history=s["history"],
                                   hist_len=s["hist_len"], repetition=s["repetition"], frequency=s["frequency"],
                                   presence=s["presence"], temperature=s["temperature"], bias=s["bias"],
                                   bias_index=s["bias_index"], allowed=s["allowed"], state=s["state"], mask=s["mask"],
                                   node_token=s["node_token"])
    x = s["logits"].float()
    rows, V = x.shape
    U = s["row_off"].numel() - 1
    row_off, hist = s["row_off"].long(), s["history"].long() - s["base"]
    user = torch.searchsorted(row_off[1:].contiguous(), torch.arange(rows, device=DEV), right=True)
    there = (hist >= 0) & (hist < V) & (torch.arange(hist.shape[1], device=DEV)[None, :] < s["hist_len"][:, None])
    count = torch.zeros((U, V), device=DEV).scatter_add_(1, hist.clamp(0, V - 1), there.float())[user]
    if s["mask"] is not None:
        T = s["node_token"].shape[1]
        node = torch.arange(T, device=DEV)
        on = ((s["mask"][:, node // 64] >> (node % 64)) & 1).float()
        count.scatter_add_(1, (s["node_token"].long() - s["base"])[user].clamp(0, V - 1), on)
    rep, freq, pres, temp = (s[k][user][:, None] for k in ("repetition", "frequency", "presence", "temperature"))
    seen = torch.where(x > 0, x / rep, x * rep) - freq * count - pres
    x = torch.where(count > 0, seen, x)
    which = s["bias_index"].long()[user]
    x = torch.where(which[:, None] >= 0, x + s["bias"][which.clamp(min=0)], x) / temp
    col = torch.arange(V, device=DEV)
    state = s["state"].long()
    fine = ((s["allowed"][state.clamp(min=0)][:, col // 32] >> (col % 32).int()) & 1).bool()
    return torch.where(fine | (state < 0)[:, None], x, -math.inf)


_RUN = dict(plan=_run_plan, append=_run_append, attention=_run_attention, rules=_run_rules)


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    if case["op"] == "plan":
        return None                                    # whole numbers
    s = prepare(case, seed)
    if case["op"] == "append":
        caches = dict(k_cache=s["k_cache"].double(), v_cache=s["v_cache"].double())
        page = case["page"]
        for r, at in enumerate(s["slot"].tolist()):
            caches["k_cache"][at // page, at % page] = s["k"][r].double()
            caches["v_cache"][at // page, at % page] = s["v"][r].double()
        return caches
    off = s["row_off"].tolist()
    if case["op"] == "rules":
        x = s["logits"].double()
        out = torch.empty_like(x)
        V, base = case["cols"], s["base"]
        bits = (1 << torch.arange(32, device=DEV)).long()
        for u in range(case["users"]):
            past = s["history"][u, :int(s["hist_len"][u])]
            rep, freq, pres, temp = (float(s[k][u]) for k in ("repetition", "frequency", "presence", "temperature"))
            for r in range(off[u], off[u + 1]):
                tokens = past
                if s["mask"] is not None:
                    path = [64 * w + b for w, bits64 in enumerate(s["mask"][r].tolist()) for b in range(64)
                            if (bits64 >> b) & 1]
                    tokens = torch.cat([past, s["node_token"][u, torch.tensor(path, device=DEV)]])
                tokens = tokens.long() - base
                n = torch.bincount(tokens[(tokens >= 0) & (tokens < V)], minlength=V).double()
                y = x[r].clone()
                y = torch.where(n > 0, torch.where(y > 0, y / rep, y * rep) - (freq * n + pres), y)
                if int(s["bias_index"][u]) >= 0:
                    y += s["bias"][int(s["bias_index"][u])].double()
                y /= temp
                if int(s["state"][r]) >= 0:
                    word = s["allowed"][int(s["state"][r])].long()
                    ok = ((word[:, None] & bits[None, :]) != 0).reshape(-1)[:V]
                    y[~ok] = -math.inf
                out[r] = y
        return out
    H, K, dh, page = case["heads"], case["kv_heads"], case["dh"], case["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for u in range(case["users"]):
        n, before = off[u + 1] - off[u], int(s["ctx"][u])
        total = before + n
        pages = s["table"][u, :-(-total // page)].long()
        k = s["k_cache"][pages].reshape(-1, K, dh)[:total].double()
        v = s["v_cache"][pages].reshape(-1, K, dh)[:total].double()
        see = torch.ones((n, total), dtype=torch.bool, device=DEV)
        if s["mask"] is None:
            see[:, before:] = torch.ones((n, n), dtype=torch.bool, device=DEV).tril()
        else:
            m = s["mask"][off[u]:off[u + 1]]
            for i in range(n):
                see[:, before + i] = (m[:, i // 64] >> (i % 64)) & 1 == 1
        for h in range(H):
            z = s["q"][off[u]:off[u + 1], h].double() @ k[:, h * K // H].T / math.sqrt(dh)
            z[~see] = -math.inf
            lse[off[u]:off[u + 1], h] = torch.logsumexp(z, -1)
            out[off[u]:off[u + 1], h] = torch.softmax(z, -1) @ v[:, h * K // H]
    return dict(out=out, lse=lse)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c, U = case, case["users"]
    if c["op"] == "plan":
        rows, pages = int(_lengths(U, c["new"]).sum()), int(_lengths(U, c["held"]).sum()) // c["page"]
        mask = 8 * _words(c["new"]) if c["tree"] else 0
        # the lengths, each row's four numbers and mask, the parents, and about a fifth of the pages changing hands
        return dict(bytes=32 * U + U * c["new"] * (16 + mask) + (4 * rows if c["tree"] else 0) + 0.2 * 8 * pages, flops=rows)
    es = 2 if c.get("dtype") == "bf16" else 4
    if c["op"] == "append":
        return dict(bytes=int(_lengths(U, c["new"]).sum()) * (4 * c["kv_heads"] * c["dh"] * es + 4), flops=0)
    if c["op"] == "rules":
        rows, V = int(_lengths(U, c["new"], c["new"] > 1).sum()), c["cols"]
        return dict(bytes=rows * V * (es + 4) + 4 * int(_lengths(U, c["hist"]).sum()) + 12 * V
                    + min(rows, c["states"]) * V / 8, flops=8 * rows * V)
    ctx, new = _lengths(U, c["ctx"], c["ragged"]), _lengths(U, c["new"], c["ragged"])
    # a tree's row sees the context and its path (about half the levels), a chain's row what stands before it
    pairs = int((new * ctx).sum()) + (int(new.sum()) * (c["levels"] + 1) / 2 if c["tree"] else int((new * (new + 1)).sum()) / 2)
    moved = (int((ctx + new).sum()) * 2 * c["kv_heads"] + int(new.sum()) * 2 * c["heads"]) * c["dh"] * es
    return dict(bytes=moved + 4 * int(new.sum()) * c["heads"], flops=4.0 * pairs * c["heads"] * c["dh"])

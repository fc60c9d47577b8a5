"""Plain implementations of the paged operators, written from their definitions in
include/atspeed.h: the step plan in Python integers, attention and logit rules in 64 bits.
Test infrastructure only."""
import math

import numpy as np
import torch


def plan(held, keep, add, table, free, n_free, page, max_rows, parent=None):
    """Sequential step plan; returns the outputs with table and free list updated (free past n_free: None)."""
    held, keep, add = (list(map(int, x)) for x in (held, keep, add))
    table, free = [list(map(int, r)) for r in table], list(map(int, free))
    B, most, pool = len(held), len(table[0]), len(free)
    words = 0 if parent is None else -(-len(parent[0]) // 64)
    off = [0]
    for a in add:
        off.append(off[-1] + max(a, 0))
    refused, before, after = [0] * B, [0] * B, [0] * B
    for b in range(B):
        before[b], after[b] = -(-held[b] // page), -(-(keep[b] + add[b]) // page)
        if (held[b] < 0 or keep[b] < 0 or keep[b] > held[b] or add[b] < 0 or before[b] > most or after[b] > most
                or keep[b] + add[b] >= 2 ** 31 or off[b + 1] > max_rows
                or (parent is not None and add[b] > len(parent[0]))):
            refused[b] = 2
    stack = free[:n_free]
    for b in range(B):
        if not refused[b]:
            stack += table[b][after[b]:before[b]]
    wanted, have = 0, len(stack)
    for b in range(B):
        want = 0 if refused[b] else max(0, after[b] - before[b])
        wanted += want
        if want and wanted > have:
            refused[b] = 1
        elif want:
            for p in range(before[b], after[b]):
                table[b][p] = stack.pop()
    free = stack + [None] * (pool - len(stack))
    length = [held[b] if refused[b] else keep[b] + add[b] for b in range(B)]
    ctx = [-1 if refused[b] else keep[b] for b in range(B)]
    rows = dict(row_user=[-1] * max_rows, row_pos=[-1] * max_rows, slot=[-1] * max_rows, tree_slot=[-1] * max_rows)
    mask = np.zeros((max_rows, words), np.uint64)
    for b in range(B):
        for r in range(off[b], min(off[b + 1], max_rows)):
            i = r - off[b]
            rows["row_user"][r] = b
            if parent is None or i < len(parent[0]):      # rows past a request's nodes are no rows of [B, max_nodes]
                rows["tree_slot"][r] = i if parent is None else b * len(parent[0]) + i
            if refused[b]:
                continue
            p = keep[b] + i
            pg = table[b][p // page]
            if 0 <= pg < pool:
                rows["slot"][r] = pg * page + p % page
            rows["row_pos"][r] = p
            if parent is not None:
                path, cur = [], i
                while cur >= 0:
                    path.append(cur)
                    up = int(parent[b][cur])
                    if up < -1 or up >= cur:
                        path = []
                        break
                    cur = up
                rows["row_pos"][r] = keep[b] + len(path) - 1 if path else -1
                for j in path:
                    mask[r, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return dict(table=table, free=free, n_free=len(stack), length=length, ctx=ctx, refused=refused,
                row_off=[min(o, max_rows) for o in off], mask=mask.view(np.int64), **rows)


def tree_parents(rng, n, levels, width):
    """A random level-ordered tree of n nodes in a row of the given width (-1 past it)."""
    parent = np.full(width, -1, np.int32)
    sizes = [len(x) for x in np.array_split(np.arange(n), max(1, min(levels, n)))]
    at = 0
    for l, m in enumerate(sizes):
        if l:
            parent[at:at + m] = rng.integers(at - sizes[l - 1], at, m)
        at += m
    return parent


def visible(ctx, count, i, total, mask_row=None):
    """Keys that the i-th new row of a request sees, of `total` keys."""
    see = np.zeros(total, bool)
    if ctx < 0:
        return see
    see[:ctx] = True
    for j in range(min(count, total - ctx)):
        on = j <= i if mask_row is None else j < 64 * len(mask_row) and (int(mask_row[j // 64]) >> (j % 64)) & 1
        see[ctx + j] = bool(on)
    return see


def attention(q, k_cache, v_cache, table, row_off, ctx, mask=None, scale=None):
    """In 64 bits on the CPU, row by row: (out, lse, spread) with spread the sum of p |v|, and the largest
    sum of |q k| of a row's visible keys."""
    q, kc, vc = (x.detach().cpu().double() for x in (q, k_cache, v_cache))
    table, row_off, ctx = (x.cpu().numpy() for x in (table, row_off, ctx))
    mask = None if mask is None else mask.cpu().numpy()
    n, H, dh = q.shape
    pool, page, K, _ = kc.shape
    scale = 1 / math.sqrt(dh) if scale is None else scale
    out, lse = torch.zeros(n, H, dh, dtype=torch.float64), torch.full((n, H), -math.inf, dtype=torch.float64)
    spread, reach = torch.zeros(n, H, dh, dtype=torch.float64), torch.zeros(n, H, dtype=torch.float64)
    heads = torch.arange(H) // (H // K)
    for b in range(len(ctx)):
        lo, hi = int(row_off[b]), min(int(row_off[b + 1]), n)
        if ctx[b] < 0 or hi <= lo:
            continue
        total = min(int(ctx[b]) + int(row_off[b + 1]) - lo, table.shape[1] * page)
        at = np.arange(total)
        pages = table[b, at // page].astype(np.int64)
        good = (pages >= 0) & (pages < pool)
        rows = torch.from_numpy(np.where(good, pages * page + at % page, 0))
        k, v = kc.reshape(-1, K, dh)[rows], vc.reshape(-1, K, dh)[rows]
        for r in range(lo, hi):
            see = torch.from_numpy(np.nonzero(visible(int(ctx[b]), int(row_off[b + 1]) - lo, r - lo, total,
                                                      None if mask is None else mask[r]) & good)[0])
            if not len(see):
                continue
            kk, vv = k[see][:, heads].permute(1, 0, 2), v[see][:, heads].permute(1, 0, 2)      # [H, n, dh]
            s = torch.bmm(kk, q[r][:, :, None])[:, :, 0] * scale
            lse[r] = torch.logsumexp(s, -1)
            p = torch.softmax(s, -1)
            out[r] = torch.bmm(p[:, None], vv)[:, 0]
            spread[r] = torch.bmm(p[:, None], vv.abs())[:, 0]
            reach[r] = (torch.bmm(kk.abs(), q[r].abs()[:, :, None])[:, :, 0] * abs(scale)).amax(-1)
    return out, lse, spread, reach


def logit_rules(logits, row_off, token_base=0, history=None, hist_len=None, repetition=None, frequency=None,
                presence=None, temperature=None, bias=None, bias_index=None, allowed=None, state=None, mask=None,
                node_token=None, mask_value=-math.inf):
    """(result, magnitude of what was added up) in 64 bits on the CPU; rows past the last request are NaN."""
    x = logits.detach().cpu().double()
    n, V = x.shape
    mask_value = float(np.float32(mask_value))        # the argument is a float
    num = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
    row_off, history, hist_len, mask, node_token, bias_index, allowed, state = map(
        num, (row_off, history, hist_len, mask, node_token, bias_index, allowed, state))
    out, size = torch.full((n, V), math.nan, dtype=torch.float64), torch.zeros(n, V, dtype=torch.float64)
    of = lambda t, b, other: other if t is None else float(t[b])  # noqa: E731
    for b in range(len(row_off) - 1):
        for r in range(int(row_off[b]), min(n, int(row_off[b + 1]))):
            tokens = []
            if history is not None:
                tokens += list(history[b, :min(max(0, int(hist_len[b])), history.shape[1])])
            if node_token is not None:
                i = r - int(row_off[b])
                tokens += [node_token[b, j] for j in range(node_token.shape[1])
                           if (j <= i if mask is None else
                               j < 64 * mask.shape[1] and (int(mask[r, j // 64]) >> (j % 64)) & 1)]
            cols = np.array(tokens, np.int64) - token_base
            count = torch.from_numpy(np.bincount(cols[(cols >= 0) & (cols < V)], minlength=V)).double()
            y = x[r].clone()
            if repetition is None and frequency is None and presence is None:
                count.zero_()
            rep, freq, pres, temp = (of(t, b, o) for t, o in ((repetition, 1.0), (frequency, 0.0), (presence, 0.0),
                                                             (temperature, 1.0)))
            y = torch.where(count > 0, torch.where(y > 0, y / rep, y * rep) - (freq * count + pres), y)
            mag = x[r].abs() * max(rep, 1 / rep) + (abs(freq) * count + abs(pres)) * (count > 0)
            w = -1 if bias is None else 0 if bias_index is None else int(bias_index[b])
            if bias is not None and 0 <= w < bias.shape[0]:
                y, mag = y + bias[w].cpu().double(), mag + bias[w].cpu().double().abs()
            y, mag = y / temp, mag / temp
            if allowed is not None and state[r] >= 0:
                s = int(state[r])
                ok = [s < allowed.shape[0] and bool((int(allowed[s, c // 32]) >> (c % 32)) & 1) for c in range(V)]
                y = torch.where(torch.tensor(ok), y, torch.full_like(y, mask_value))
            out[r], size[r] = y, mag
    return out, size

"""Plain implementations, from the definitions in include/atspeed.h, of beam selection and
distillation in 64 bits and of forked pages in Python integers.  Test infrastructure only."""
import math

import numpy as np


# ---------------------------------------------------------------- beam selection

def select(logits, row_off, k, score=None, done=None, token_base=0, log_probs=False, row_id=None, paths=None,
           path_len=None):
    """logits: float64 [rows, cols].  Returns count, parent, token, score (float64) and the grown paths, as lists."""
    rows, cols = logits.shape
    out = dict(count=[], parent=[], token=[], score=[], paths=[], path_len=[])
    end = min(int(row_off[-1]), rows)
    for b in range(len(row_off) - 1):
        cand = []
        for r in range(max(int(row_off[b]), 0), min(int(row_off[b + 1]), end)):
            s = 0.0 if score is None else float(score[r])
            if not math.isfinite(s):
                continue
            if done is not None and done[r]:
                cand.append((-s, r, -1))
                continue
            x = logits[r]
            if np.isnan(x).any() or (x == math.inf).any() or not (x > -math.inf).any():
                continue
            top = x.max()
            # the largest logit is taken from the others before the score comes in: beside a logit of 3e38 a score is lost
            z = s + x if log_probs else (s - math.log(np.exp(x - top).sum())) + (x - top)
            best = np.lexsort((np.arange(cols), -z))[:k]
            cand += [(-z[v], r, int(v)) for v in best if x[v] > -math.inf]
        cand = sorted(cand)[:k]
        pad = k - len(cand)
        name = lambda r: r if row_id is None else int(row_id[r])  # noqa: E731
        out["count"].append(len(cand))
        out["parent"].append([name(r) for _, r, _ in cand] + [-1] * pad)
        out["token"].append([-1 if v < 0 else token_base + v for _, _, v in cand] + [-1] * pad)
        out["score"].append([-s for s, _, _ in cand] + [-math.inf] * pad)
        if paths is not None:
            most, grown = len(paths[0]), []
            for _, r, v in cand:
                known = 0 <= name(r) < len(paths)
                p = list(paths[name(r)][:min(max(int(path_len[name(r)]), 0), most)]) if known else []
                if v >= 0 and len(p) < most:
                    p.append(token_base + v)
                grown.append([int(t) for t in p])
            out["path_len"].append([len(p) for p in grown] + [0] * pad)
            out["paths"].append([p + [-1] * (most - len(p)) for p in grown] + [[-1] * most] * pad)
    return out


# ---------------------------------------------------------------- forked pages

def fork(held, keep, table, free, n_free, shared, page, src=None):
    """Rows one after the other.  Returns the outputs and the state; None where it is undefined."""
    held, table, shared = [int(h) for h in held], [[int(p) for p in r] for r in table], [int(x) for x in shared]
    B, most, pool = len(held), len(table[0]), len(shared)
    held = [h if 0 <= h <= most * page else 0 for h in held]
    src = list(range(B)) if src is None else [int(s) for s in src]
    refused, kept = [0] * B, [0] * B
    for j in range(B):
        there = held[src[j]] if 0 <= src[j] < B else 0
        kept[j] = 0 if src[j] == -1 else there if keep is None else int(keep[j])
        if not -1 <= src[j] < B or not 0 <= kept[j] <= there:
            refused[j], src[j], kept[j] = 2, j, held[j]
    sound = lambda p: 0 <= p < pool  # noqa: E731
    full, over = [c // page for c in kept], [c % page for c in kept]
    old = [p for j in range(B) for p in table[j][:-(-held[j] // page)] if sound(p)]
    outside = list(shared)                                   # holders that are no rows, less one
    for p in old:
        outside[p] -= 1
    stays = [0] * pool
    for j in range(B):
        for p in table[src[j]][:full[j]] if src[j] >= 0 else []:
            if sound(p):
                stays[p] += 1
    takes, wants = [False] * B, []
    taken = set()
    for j in range(B):
        if src[j] < 0 or not over[j] or not sound(table[src[j]][full[j]]):
            continue
        p = table[src[j]][full[j]]
        if stays[p] == 0 and outside[p] < 0 and p not in taken:
            takes[j] = True
            taken.add(p)
        else:
            wants.append(j)
    gone = []
    for p in sorted(set(old)):
        left = outside[p] + stays[p] + (p in taken)
        shared[p] = max(left, 0)
        if left < 0 and p not in taken:
            gone.append(p)
    stack = [int(p) for p in free[:n_free]] + gone
    copies = [(-1, -1, 0)] * B
    length = list(kept)
    new = [list(r) for r in table]
    for j in range(B):
        if src[j] >= 0:
            last = full[j] + (1 if over[j] and j not in wants else 0)
            new[j][:last] = table[src[j]][:last]
    for j in wants:
        if stack:
            p = stack.pop()
            copies[j] = (table[src[j]][full[j]], p, over[j])
            new[j][full[j]] = p
        else:
            refused[j], length[j] = refused[j] or 1, full[j] * page
    for j in range(B):
        for c in range(-(-length[j] // page), most):
            new[j][c] = None
    return dict(table=new, free=stack + [None] * (pool - len(stack)), n_free=len(stack), shared=shared, length=length,
                refused=refused, copy_src=[c[0] for c in copies], copy_dst=[c[1] for c in copies],
                copy_len=[c[2] for c in copies])


# ---------------------------------------------------------------- distillation

EPS = 2.0 ** -24


def distill(logits, teacher, index, tail=None, weight=None, T=1.0, reverse=False, grad_loss=None):
    """float64 loss [rows], gradient [rows, cols], and what fp32 arithmetic may move them by.

    The bounds count roundings (EPS each): an exponential exp2((z - top) * c) has the roundings of the difference, of c
    and of the product, 3 EPS of its argument, and two of its own; a sum of a row's exponentials in vectors adds up to
    10 + cols / 1024 of them and a product for each time a thread's largest moves.
    """
    rows, cols = logits.shape
    loss, grad = np.zeros(rows), np.zeros((rows, cols))
    loss_off, grad_off = np.zeros(rows), np.zeros((rows, cols))
    for r in range(rows):
        w = 1.0 if weight is None else float(weight[r])
        g = 1.0 if grad_loss is None else float(grad_loss[r])
        tops = {}
        entries = [(int(v), float(t)) for v, t in zip(index[r], teacher[r]) if 0 <= v < cols and t != -math.inf]
        if not entries or w == 0.0:
            continue
        rest_t = -math.inf if tail is None else float(tail[r])
        t_top = max([t / T for _, t in entries] + [rest_t])
        total = sum(math.exp(t / T - t_top) for _, t in entries) + math.exp(rest_t - t_top)
        for v, t in entries:
            tops[v] = tops.get(v, 0.0) + math.exp(t / T - t_top) / total
        p_rest = math.exp(rest_t - t_top) / total
        # log p without p, which is 0 from 745 below the largest on: around the largest entry of each bucket
        log_p, log_p_rest = {}, (rest_t - t_top) - math.log(total)
        for v in tops:
            mine = [t / T for u, t in entries if u == v]
            log_p[v] = (max(mine) - t_top) + math.log(sum(math.exp(t - max(mine)) for t in mine)) - math.log(total)
        cols_of = np.array(sorted(tops))
        p = np.array([tops[v] for v in cols_of])
        others = np.ones(cols, bool)
        others[cols_of] = False
        z = logits[r] / T
        top = z.max()
        d = z - top if top > -math.inf else np.full(cols, -math.inf)
        e = np.exp(d)
        finite = np.where(np.isfinite(d), np.abs(d), 0.0)
        err = (3 * finite + 3) * EPS                          # relative, of each exponential
        if e.sum() == 0:
            q, q_rest, rel, rel_rest = e, 0.0, 0.0, 0.0
            log_q = np.full(cols, -math.inf)
        else:
            add = (16 + cols / 1024) * EPS
            q, q_rest = e / e.sum(), e[others].sum() / e.sum()
            rel = (e * err).sum() / e.sum() + add
            rel_rest = ((e * err)[others].sum() / e[others].sum() if q_rest > 0 else 0.0) + add
            log_q = d - math.log(e.sum())
        with np.errstate(divide="ignore", invalid="ignore"):
            lp, lq = np.array([log_p[v] for v in cols_of]), log_q[cols_of]
            lpr = log_p_rest
            lqr = math.log(q_rest) if q_rest > 0 else -math.inf
            step = w * T
            qt = q[cols_of]
            d_log = 2 * finite[cols_of] * EPS + rel           # of log q at a top, and of the rest
            d_rest = rel_rest + rel
            if reverse:
                far = np.where(qt > 0, lq - lp, 0.0)
                far_r = lqr - lpr if q_rest > 0 else 0.0
                L = (qt * far).sum() + (q_rest * far_r if q_rest > 0 else 0.0)
                L_off = (qt * (np.abs(far) * (err[cols_of] + rel) + d_log)).sum() + q_rest * (abs(far_r) + 1) * d_rest
                grad[r] = step * q * (far_r - L)
                grad[r, cols_of] = step * qt * (far - L)
                grad_off[r] = step * q * (abs(far_r - L) * (err + rel) + d_rest + L_off)
                grad_off[r, cols_of] = step * qt * (np.abs(far - L) * (err[cols_of] + rel) + d_log + L_off)
            else:
                terms = np.where(p > 0, p * (lp - lq), 0.0)
                L = terms.sum() + (p_rest * (lpr - lqr) if p_rest > 0 else 0.0)
                L_off = (p * d_log).sum() + p_rest * d_rest
                share = p_rest / q_rest if q_rest > 0 else 0.0
                grad[r] = step * q * (1 - share)
                grad[r, cols_of] = step * (qt - p)
                grad_off[r] = step * q * (abs(1 - share) * (err + rel) + share * d_rest)
                grad_off[r, cols_of] = step * qt * (err[cols_of] + rel)
        loss[r] = step * T * L
        loss_off[r] = step * T * L_off + 2 * EPS * abs(loss[r]) if math.isfinite(L) else 0.0
        grad[r] *= g
        grad_off[r] = abs(g) * grad_off[r] + 4 * EPS * np.abs(grad[r])
    return loss, grad, loss_off, grad_off

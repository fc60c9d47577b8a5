"""The paged operators as they are used together: over the engine's own activations they
give the engine's attention, and a verify of the engine's drafted trees on a target that
the engine does not hold (grouped heads, histories of different lengths, paged caches,
logit rules) accepts what the same target in 64 bits accepts."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from _gpu_common import LOGIT_TOL, env  # noqa: E402
from test_gpu_paged import close_to_exact, ints  # noqa: E402
from paper_2410_05165_amd.binding import Engine  # noqa: E402
from paper_2410_05165_amd.paged import PagedKV, atspeed_logit_rules  # noqa: E402

DEV = "cuda:0"


class Captured:
    """bf16 activations of one target forward: q, k, v and the attention output per layer."""

    def __init__(self, eng, rows, fn):
        m = eng.w.target
        self.d, self.f, self.R, self.H = m.d_model, m.d_ffn, rows, m.n_heads
        self.layer = rows * (6 * self.d + self.f)
        x = torch.zeros((2 * m.n_layers + 1, rows, self.d), device=DEV)
        self.act = torch.zeros(m.n_layers * self.layer + rows * self.d, dtype=torch.int16, device=DEV)
        plan = torch.full((3 * rows + 1,), -2, dtype=torch.int32, device=DEV)
        eng.atspeed_capture_hidden(x, plan, rows, act=self.act)
        fn()
        torch.cuda.synchronize()
        p = plan.cpu().numpy()
        self.M = int(p[3 * rows])
        assert self.M <= rows
        self.user, self.pos, self.slot = p[:3 * rows].reshape(3, rows)[:, :self.M]

    def take(self, layer, part, index):
        a = self.act[layer * self.layer + part * self.R * self.d:][:self.R * self.d].view(torch.bfloat16)
        return a.view(self.R, self.H, self.d // self.H)[index]


def test_the_engines_activations_give_the_engines_attention():
    e = env("small")
    w, B, P = e["w"], e["w"].batch, e["w"].prefix_len
    eng = Engine(w, e["tw"], e["dw"], e["cat"])
    prefix = torch.from_numpy(e["pre"]).to(DEV)
    pre = Captured(eng, B * P, lambda: eng.atspeed_prefill(prefix))
    eng.atspeed_draft()
    T = eng.max_nodes
    logits = torch.zeros((B, T, w.n_item_tokens), device=DEV)
    tree = Captured(eng, B * T, lambda: eng.atspeed_tree_logits(logits))
    nodes, token, parent, depth, _ = eng.tree_tensors(B)
    parent = torch.where(torch.arange(T, device=DEV)[None] < nodes[:, None], parent, -1).contiguous()
    # the forwarded nodes: all above the last level (level order: the first ones)
    d, n = depth.cpu().numpy(), nodes.cpu().numpy()
    fwd = np.array([int((d[u, :n[u]] < w.L).sum()) for u in range(B)])
    assert fwd.sum() == tree.M

    row = {}
    for i, (u, p) in enumerate(zip(pre.user, pre.pos)):
        row[int(u), int(p)] = i
    first = torch.tensor([row.get((u, p), row.get((0, p))) for u in range(B) for p in range(P)], device=DEV)
    m = w.target
    cache = PagedKV(m.n_layers, B * (-(-(P + T) // 16)), 16, m.n_heads, m.d_head, B, P + T)
    chunk = cache.plan(ints([0] * B), ints([P] * B), B * P)
    layers = (0, m.n_layers - 1)
    worst = 0.0
    for l in layers:
        q, k, v, ao = (pre.take(l, part, first) for part in (1, 2, 3, 4))
        cache.append(l, chunk, k.contiguous(), v.contiguous())
        c = dict(q=q.contiguous(), k_cache=cache.k[l], v_cache=cache.v[l], block_table=cache.block_table,
                 row_off=chunk.row_off, ctx=chunk.ctx, max_ctx=0, max_new=P, mask=None)
        out = cache.attention(l, chunk, c["q"], P)
        if l == 0:
            close_to_exact(c, out, None)
            close_to_exact(c, ao, None)
        worst = max(worst, float((out.float() - ao.float()).abs().max()))
    step = cache.plan(ints([P] * B), ints(fwd), int(fwd.sum()), parent)
    assert int(step.refused.abs().sum()) == 0
    index = {int(s): i for i, s in enumerate(tree.slot)}
    where = torch.tensor([index[int(s)] for s in step.tree_slot], device=DEV)
    np.testing.assert_array_equal(step.row_pos.cpu().numpy(), tree.pos[where.cpu().numpy()])
    np.testing.assert_array_equal(step.row_user.cpu().numpy(), tree.user[where.cpu().numpy()])
    for l in layers:
        q, k, v, ao = (tree.take(l, part, where) for part in (1, 2, 3, 4))
        cache.append(l, step, k, v)
        c = dict(q=q, k_cache=cache.k[l], v_cache=cache.v[l], block_table=cache.block_table, row_off=step.row_off,
                 ctx=step.ctx, max_ctx=P, max_new=int(fwd.max()), mask=step.mask)
        out = cache.attention(l, step, q, int(fwd.max()), P)
        if l == 0:
            close_to_exact(c, out, None)
            close_to_exact(c, ao, None)
        worst = max(worst, float((out.float() - ao.float()).abs().max()))
    print(f"[paged] largest distance from the engine's attention: {worst:.2e}", flush=True)
    eng.close()


class Target:
    """A decoder with grouped heads in plain torch: RMSNorm, rotary attention, a gated MLP, an item head."""

    def __init__(self, seed, vocab, n_item, d=256, heads=8, kv=2, dh=64, f=512, layers=2):
        g = torch.Generator(device=DEV).manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device=DEV) / math.sqrt(s[-1])  # noqa: E731
        self.heads, self.kv, self.dh = heads, kv, dh
        self.emb, self.head = torch.randn((vocab, d), generator=g, device=DEV), r(n_item, d) * 2
        self.layers = [dict(q=r(heads * dh, d), k=r(kv * dh, d), v=r(kv * dh, d), o=r(d, heads * dh), gate=r(f, d),
                            up=r(f, d), down=r(d, f)) for _ in range(layers)]

    def rope(self, x, pos):
        half = self.dh // 2
        ang = pos[:, None].double() * (10000.0 ** (-torch.arange(half, device=DEV).double() / half))
        c, s = (t.to(x.dtype)[:, None] for t in (ang.cos(), ang.sin()))
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    def forward(self, tokens, pos, attend):
        """Logits of rows with these tokens and positions; attend(layer, q, k, v) -> [rows, heads, dh]."""
        norm = lambda x: x / x.pow(2).mean(-1, keepdim=True).add(1e-6).sqrt()  # noqa: E731
        x = self.emb.to(self.dtype)[tokens]
        for l, w in enumerate(self.layers):
            W = {n: t.to(self.dtype) for n, t in w.items()}
            y = norm(x)
            q, k, v = (y @ W[n].T for n in "qkv")
            q = self.rope(q.view(-1, self.heads, self.dh), pos)
            k = self.rope(k.view(-1, self.kv, self.dh), pos)
            x = x + attend(l, q, k, v.view(-1, self.kv, self.dh)).reshape(len(tokens), -1) @ W["o"].T
            y = norm(x)
            x = x + (torch.nn.functional.silu(y @ W["gate"].T) * (y @ W["up"].T)) @ W["down"].T
        return norm(x) @ self.head.to(self.dtype).T

    dtype = torch.float32

    def exact_logits(self, tokens):
        """The last token's logits of one sequence in 64 bits."""
        self.dtype = torch.float64
        n = len(tokens)
        ok = torch.ones((n, n), dtype=torch.bool, device=DEV).tril()

        def attend(l, q, k, v):
            k, v = (t.repeat_interleave(self.heads // self.kv, 1) for t in (k, v))
            s = torch.einsum("qhd,khd->hqk", q, k) / math.sqrt(self.dh)
            return torch.einsum("hqk,khd->qhd", torch.softmax(s.masked_fill(~ok, -math.inf), -1), v)

        out = self.forward(torch.tensor(tokens, device=DEV), torch.arange(n, device=DEV), attend)[-1]
        self.dtype = torch.float32
        return out


def test_verify_on_a_target_of_ones_own():
    e = env("tiny", batch=3)
    w, B = e["w"], 3
    n_item, base = w.n_item_tokens, w.target.item_base
    engines = [Engine(w, e["tw"], e["dw"], e["cat"]) for _ in range(2)]
    prefix = torch.from_numpy(e["pre"]).to(DEV)
    for eng in engines:
        eng.atspeed_prefill(prefix)
        eng.atspeed_draft()
    eng = engines[0]
    T = eng.max_nodes
    nodes, token, parent, depth, _ = eng.tree_tensors(B)
    n, tok, par, dep = (t.cpu().numpy() for t in (nodes, token, parent, depth))
    fwd = np.array([int((dep[u, :n[u]] < w.L).sum()) for u in range(B)])
    live = torch.arange(T, device=DEV)[None] < nodes[:, None]
    parent, token = torch.where(live, parent, -1).contiguous(), torch.where(live, token, 0).contiguous()

    # the own target sees histories of different lengths, prefilled in two chunks
    tgt = Target(5, w.target.vocab, n_item)
    hist = [e["pre"][u][: w.prefix_len - 13 * u] for u in range(B)]
    lens = np.array([len(h) for h in hist])
    cache = PagedKV(2, 64, 8, tgt.kv, tgt.dh, B, w.prefix_len + T, dtype=torch.float32)
    rules = dict(token_base=base, history=ints(np.stack([np.pad(h, (0, w.prefix_len - len(h))) for h in hist])),
                 hist_len=ints(lens), repetition=torch.full((B,), 1.2, device=DEV),
                 presence=torch.full((B,), 0.1, device=DEV), temperature=torch.full((B,), 0.9, device=DEV))
    rng = np.random.default_rng(3)
    ban = rng.random((2, n_item)) < 0.02              # codes that may not be recommended, per group of users
    words = np.packbits(~ban, axis=-1, bitorder="little").view(np.int32)
    rules["allowed"] = ints(words)
    low = -1.0e4                                       # a finite value: acceptance takes its log-softmax

    def run(plan, tokens, rows, width):
        def attend(l, q, k, v):
            cache.append(l, plan, k, v)
            return cache.attention(l, plan, q, width)
        return tgt.forward(tokens, plan.row_pos[:rows].long(), attend)

    cut, root = lens // 3, None
    for lo, hi in ((np.zeros(B, int), cut), (cut, lens)):
        add = hi - lo
        plan = cache.plan(ints(lo), ints(add), int(add.sum()))
        toks = torch.from_numpy(np.concatenate([hist[u][lo[u]:hi[u]] for u in range(B)])).to(DEV).long()
        z = run(plan, toks, int(add.sum()), int(add.max()))
        root = z[plan.row_off[1:].long() - 1].contiguous()
    one = ints(np.arange(B + 1))
    group = ints(np.arange(B) % 2)
    root = atspeed_logit_rules(root, one, state=group, mask_value=low, **rules)

    rows = int(fwd.sum()) + 5                           # five rows of padding behind the last request
    step = cache.plan(ints(lens), ints(fwd), rows, parent)
    assert int(step.refused.abs().sum()) == 0
    toks = torch.where(step.tree_slot >= 0, token.view(-1)[step.tree_slot.clamp(min=0).long()], 0).long()
    z = run(step, toks, rows, int(fwd.max()))
    state = torch.where(step.row_user >= 0, group[step.row_user.clamp(min=0).long()], -1).int()
    logits = torch.zeros((B, T, n_item), device=DEV)
    atspeed_logit_rules(z, step.row_off, out=logits, out_row=step.tree_slot, state=state, mask=step.mask,
                        node_token=token, mask_value=low, **rules)

    # the same in 64 bits, a whole forward for each node
    def exact(u, path):
        x = tgt.exact_logits(np.concatenate([hist[u], np.array(path, np.int32)]).astype(np.int64))
        seen = np.bincount(np.concatenate([hist[u], path]).astype(np.int64) - base, minlength=n_item)[:n_item] > 0
        y = x.cpu().numpy()
        y = np.where(seen, np.where(y > 0, y / np.float64(np.float32(1.2)), y * np.float64(np.float32(1.2)))
                     - np.float64(np.float32(0.1)), y) / np.float64(np.float32(0.9))
        return np.where(ban[u % 2], low, y)

    want_root, want = np.stack([exact(u, []) for u in range(B)]), np.zeros((B, T, n_item))
    for u in range(B):
        for i in range(fwd[u]):
            path, j = [], i
            while j >= 0:
                path.insert(0, int(tok[u, j]))
                j = int(par[u, j])
            want[u, i] = exact(u, path)
            assert np.abs(logits[u, i].cpu().numpy() - want[u, i]).max() <= LOGIT_TOL["fp32"]
    assert np.abs(root.cpu().numpy() - want_root).max() <= LOGIT_TOL["fp32"]
    engines[0].atspeed_accept(logits, root)
    engines[1].atspeed_accept(torch.from_numpy(want).float().to(DEV), torch.from_numpy(want_root).float().to(DEV))
    a, b = (x.atspeed_get_state(B) for x in engines)
    np.testing.assert_array_equal(a[0], b[0])
    for u in range(B):
        t, k = int(a[0][u]), int(a[1][u])
        assert t >= 1 and k == int(b[1][u])
        np.testing.assert_array_equal(a[2][u, :k, :t], b[2][u, :k, :t])
        for path in a[2][u, :k, :t]:
            assert not any(ban[u % 2][w.codebook * l + c] for l, c in enumerate(path))
    # next step: the accepted length goes on, the drafted rows' pages come back
    before = int(cache.n_free)
    cache.plan(ints(lens), ints([0] * B), 0)
    assert int(cache.n_free) >= before and cache.length.cpu().tolist() == lens.tolist()
    for x in engines:
        x.close()

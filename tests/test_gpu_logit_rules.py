"""Logit rules on the engine's own forwards (atspeed_set_logit_rules): a decode under rules
gives the lists of the oracle's beam search whose log-probs the rules changed, the same
lists as the target-only search under them, and without rules what it gave before."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from _gpu_common import SCORE_TOL, env  # noqa: E402
from oracle.model import Decoder  # noqa: E402
from oracle.search import Scorer, beam_search, model_scorer  # noqa: E402
from paper_2410_05165_amd.binding import AlignArgs, AtspeedError, Engine  # noqa: E402

DEV = "cuda:0"


def gpu(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).to(DEV)


def make_rules(w, cat, seed, B):
    """Bans of the most frequent first codes, code biases, temperatures and penalties for codes of the history."""
    rng = np.random.default_rng(seed)
    n, cb = w.n_item_tokens, w.codebook
    top = np.argsort(-np.bincount(cat[:, 0], minlength=cb))[:40]
    allowed = np.ones((2, (n + 31) // 32 * 32), bool)
    allowed[0, top] = False
    allowed[1, cb:2 * cb] = rng.random(cb) < 0.7
    host = dict(history=rng.integers(0, n, (B, 25)) + w.target.item_base, hist_len=rng.integers(0, 26, B),
                presence=rng.uniform(0, 0.4, B), frequency=rng.uniform(0, 0.2, B), temperature=rng.uniform(0.6, 1.4, B),
                bias=rng.standard_normal((2, n)) * 0.3, bias_index=np.arange(B) % 3 - 1, state=np.arange(B) % 3 - 1)
    kinds = dict(history=np.int32, hist_len=np.int32, bias_index=np.int32, state=np.int32)
    dev = {k: gpu(v, kinds.get(k, np.float32)) for k, v in host.items()}
    dev["allowed"] = gpu(np.packbits(allowed, axis=-1, bitorder="little").view(np.int32), np.int32)
    host = {k: v.astype(np.float32).astype(np.float64) if v.dtype == np.float64 else v for k, v in host.items()}
    return dev, dict(host, allowed=allowed[:, :n])


def ruled(lp, h, u, w):
    """The scorer of a user under the rules (a log-softmax row differs from its logits by a constant)."""
    n = w.n_item_tokens
    count = np.bincount(h["history"][u, :h["hist_len"][u]] - w.target.item_base, minlength=n).astype(float)

    def fn(paths):
        out = []
        for row in lp(paths):
            x = row - np.where(count > 0, h["frequency"][u] * count + h["presence"][u], 0.0)
            if h["bias_index"][u] >= 0:
                x = x + h["bias"][h["bias_index"][u]]
            x = x / h["temperature"][u]
            if h["state"][u] >= 0:
                x = np.where(h["allowed"][h["state"][u]], x, -1.0e4)
            x = x - x.max()
            out.append(x - np.log(np.exp(x).sum()))
        return np.stack(out)
    return Scorer(fn)


def decode(eng, w, prefix, search=False):
    B = prefix.shape[0]
    items = torch.zeros((B, w.K, w.L), dtype=torch.int32, device=DEV)
    scores, n = torch.zeros((B, w.K), device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    (eng.atspeed_target_search if search else eng.atspeed_decode_topk)(prefix, items, scores, n)
    torch.cuda.synchronize()
    return items.cpu().numpy(), scores.cpu().numpy(), n.cpu().numpy()


@pytest.mark.parametrize("reuse,start", [(0, 0), (1, 1)])
def test_ruled_decode_equals_the_oracles_ruled_search(reuse, start):
    e = env("tiny", batch=4)
    w, B = e["w"], 4
    eng = Engine(w, e["tw"], e["dw"], e["cat"], reuse_tree_kv=reuse, sd_start_level=start)
    prefix = torch.from_numpy(e["pre"]).to(DEV)
    plain = decode(eng, w, prefix)
    dev, host = make_rules(w, e["cat"], 1, B)
    eng.atspeed_set_logit_rules(**dev)
    with pytest.raises(AtspeedError) as ex:
        eng.atspeed_draft()                              # the batch ended with the rules
    assert ex.value.status == 5
    got, searched = decode(eng, w, prefix), decode(eng, w, prefix, search=True)
    for a, b in zip(got, searched):
        np.testing.assert_array_equal(a, b)
    tgt = Decoder(w.target, e["tw"], w.dtype)
    for u in range(B):
        lp = ruled(model_scorer(tgt, tgt.prefill(e["pre"][u]), w.target.item_base, w.codebook), host, u, w)
        want = beam_search(lp, e["trie"], w.K, w.L, w.codebook)[-1]
        assert [tuple(r) for r in got[0][u].tolist()] == [p for p, _ in want], u
        np.testing.assert_allclose(got[1][u], [s for _, s in want], rtol=0, atol=SCORE_TOL)
        if host["state"][u] >= 0:
            ok = host["allowed"][host["state"][u]]
            assert all(ok[w.codebook * l + c] for r in got[0][u] for l, c in enumerate(r))
        # a temperature and a few penalties may leave an order as it was; biases of 0.3 a code do not
        assert host["bias_index"][u] < 0 or not np.array_equal(got[0][u], plain[0][u])
    eng.atspeed_set_logit_rules()
    for a, b in zip(plain, decode(eng, w, prefix)):
        np.testing.assert_array_equal(a, b)
    eng.close()


def test_neutral_rules_change_nothing():
    e = env("tiny", batch=4)
    w = e["w"]
    eng = Engine(w, e["tw"], e["dw"], e["cat"])
    prefix = torch.from_numpy(e["pre"]).to(DEV)
    plain = decode(eng, w, prefix)
    one = torch.ones(4, device=DEV)
    eng.atspeed_set_logit_rules(history=gpu(np.zeros((4, 3)), np.int32), hist_len=gpu([0, 3, 1, 2], np.int32),
                                repetition=one, frequency=0 * one, presence=0 * one, temperature=one,
                                bias=torch.zeros((1, w.n_item_tokens), device=DEV),
                                allowed=gpu(np.full((1, (w.n_item_tokens + 31) // 32), -1), np.int32),
                                state=gpu([0, -1, 0, 0], np.int32))
    for a, b in zip(plain, decode(eng, w, prefix)):
        np.testing.assert_array_equal(a, b)
    eng.close()


@pytest.mark.parametrize("name,mode", [("small", 2), ("tiny", 1), ("tiny", 2)])
def test_relaxed_decode_keeps_to_the_rules(name, mode):
    e = env(name)
    w, B = e["w"], e["w"].batch
    eng = Engine(w, e["tw"], e["dw"], e["cat"], mode=mode, seed=3)
    dev, host = make_rules(w, e["cat"], 2, B)
    eng.atspeed_set_logit_rules(**dev)
    items, _, n = decode(eng, w, torch.from_numpy(e["pre"]).to(DEV))
    for u in range(B):
        assert n[u] > 0
        if host["state"][u] >= 0:
            ok = host["allowed"][host["state"][u]]
            assert all(ok[w.codebook * l + c] for r in items[u, :n[u]] for l, c in enumerate(r)), u
    eng.close()


def test_refusals():
    e = env("tiny", batch=4)
    w = e["w"]
    eng = Engine(w, e["tw"], e["dw"], e["cat"])
    one = torch.ones(4, device=DEV)
    for kw, status in ((dict(mask_value=-float("inf")), 1), (dict(history=gpu(np.zeros((4, 3)), np.int32)), 1),
                       (dict(allowed=gpu(np.zeros((1, (w.n_item_tokens + 31) // 32)), np.int32)), 1)):
        with pytest.raises(AtspeedError) as ex:
            eng.atspeed_set_logit_rules(**kw)
        assert ex.value.status == status
    for kw in (dict(temperature=one[:3]), dict(bias=torch.zeros((1, 5), device=DEV)), dict(presence=one.double())):
        with pytest.raises(ValueError):
            eng.atspeed_set_logit_rules(**kw)
    prefix = torch.from_numpy(e["pre"]).to(DEV)
    eng.atspeed_set_logit_rules(temperature=one)
    eng.atspeed_prefill(prefix)
    items = gpu(np.repeat(e["cat"][None, :2], 4, 0), np.int32)
    args = AlignArgs()
    for f in ("ctx_weight", "label_weight", "root_weight", "log_pK", "lp_target", "root_target", "master", "adam_m",
              "adam_v", "grad"):
        setattr(args, f, one.data_ptr())                 # refused before any of them is looked at
    args.step, args.eps = 1, 1e-8
    for call in (lambda: eng.atspeed_align_data(items, None, gpu([2] * 4, np.int32), args), lambda: eng.atspeed_align_step(args)):
        with pytest.raises(AtspeedError) as ex:
            call()
        assert ex.value.status == 5
    eng.close()

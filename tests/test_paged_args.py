"""The context-free paged calls: their structures match the header, and every argument
error is found on the host before any launch (no GPU needed)."""
import ctypes as C
import os
import re

import pytest

from paper_2410_05165_amd import binding as bd

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "atspeed.h")
P = 0x10000      # an aligned address that nothing reads: every call below ends on the host
OK, INVALID, SHAPE, WORKSPACE = 0, 1, 2, 3


@pytest.mark.parametrize("cls,name", [(bd.PagePlanArgs, "atspeed_page_plan_args"), (bd.KvAppendArgs, "atspeed_kv_append_args"),
                                      (bd.TreeAttentionArgs, "atspeed_tree_attention_args"),
                                      (bd.LogitRulesArgs, "atspeed_logit_rules_args")])
def test_structures_follow_the_header(cls, name):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", text).group(1)
    kinds = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float}
    want = []
    for line in filter(None, (x.strip() for x in body.split(";"))):
        kind, names = re.match(r"((?:const )?\w+\s*\*?)\s*(.*)", line, re.S).groups()
        for n in (x.strip() for x in names.split(",")):
            if kind.strip() == "atspeed_pages":
                s = n.split("_")[0]
                want += [(s + "_data", C.c_void_p)] + [(f"{s}_{x}", C.c_int64) for x in ("page", "token", "head")]
            else:
                want.append((n, C.c_void_p if "*" in kind else kinds[kind.strip()]))
    assert want == [(n, t) for n, t in cls._fields_]


def fill(cls, **kw):
    a = cls()
    at = P
    for n, t in cls._fields_:
        if t is C.c_void_p:
            at += 1 << 20
            setattr(a, n, at)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def refuse(call, cls, good, bad, *more):
    lib = bd.load_library()
    for status, kw in bad:
        got = getattr(lib, call)(C.byref(fill(cls, **{**good, **kw})), *more, None)
        assert got == status, (kw, got, lib.atspeed_last_error())
        assert lib.atspeed_last_error()
    assert getattr(lib, call)(None, *more, None) == INVALID


def test_plan_refusals():
    good = dict(B=4, page_size=16, max_pages=8, n_pool=40, max_rows=50, max_nodes=20)
    bad = [(INVALID, dict(B=0)), (INVALID, dict(B=1025)), (INVALID, dict(page_size=0)), (INVALID, dict(page_size=24)),
           (INVALID, dict(page_size=2048)), (INVALID, dict(n_pool=0)), (SHAPE, dict(n_pool=2 ** 27)),
           (INVALID, dict(max_pages=0)), (SHAPE, dict(B=1024, max_pages=2 ** 21)), (INVALID, dict(max_rows=-1)),
           (INVALID, dict(max_nodes=0)), (INVALID, dict(max_nodes=4097)), (INVALID, dict(mask=None))]
    bad += [(INVALID, {n: None}) for n in ("held", "keep", "add", "block_table", "free_pages", "n_free", "n_free_out",
                                           "length", "ctx", "refused", "row_off", "row_user", "row_pos", "slot",
                                           "tree_slot")]
    bad += [(INVALID, dict(length=P, held=P)), (INVALID, dict(n_free=P, n_free_out=P)), (INVALID, dict(ctx=P, keep=P))]
    refuse("atspeed_page_plan", bd.PagePlanArgs, good, bad)


def test_append_refusals():
    good = dict(dtype=bd.BF16, n_rows=3, n_kv_heads=2, d_head=128, page_size=16, n_pool=10, k_row_stride=256,
                k_head_stride=128, v_row_stride=256, v_head_stride=128, k_page=4096, k_token=256, k_head=128, v_page=4096,
                v_token=256, v_head=128)
    bad = [(INVALID, dict(dtype=2)), (SHAPE, dict(d_head=32)), (SHAPE, dict(d_head=96)), (SHAPE, dict(d_head=256)),
           (INVALID, dict(n_rows=-1)), (INVALID, dict(n_kv_heads=0)), (INVALID, dict(page_size=3)),
           (INVALID, dict(k_row_stride=260)), (INVALID, dict(v_head_stride=4)), (INVALID, dict(k_page=4097)),
           (INVALID, dict(v_token=2)), (INVALID, dict(k=P + 8)), (INVALID, dict(v_data=P + 2))]
    bad += [(INVALID, {n: None}) for n in ("k", "v", "k_data", "v_data", "slot")]
    refuse("atspeed_kv_append", bd.KvAppendArgs, good, bad)
    assert bd.load_library().atspeed_kv_append(C.byref(fill(bd.KvAppendArgs, **{**good, "n_rows": 0})), None) == OK


ATTN = dict(dtype=bd.BF16, B=2, n_rows=9, n_heads=8, n_kv_heads=2, d_head=128, page_size=16, max_pages=5, n_pool=10,
            max_ctx=70, max_new=6, mask_words=1, scale=0.1, q_row_stride=1024, q_head_stride=128, out_row_stride=1024,
            out_head_stride=128, k_page=4096, k_token=256, k_head=128, v_page=4096, v_token=256, v_head=128)


def test_attention_refusals():
    bad = [(INVALID, dict(dtype=-1)), (SHAPE, dict(d_head=32)), (SHAPE, dict(dtype=bd.FP32, d_head=16)),
           (INVALID, dict(B=0)), (INVALID, dict(B=2000)), (INVALID, dict(n_rows=-1)), (INVALID, dict(max_ctx=-1)),
           (INVALID, dict(max_new=-1)), (SHAPE, dict(n_heads=7)), (SHAPE, dict(n_heads=0)), (SHAPE, dict(n_kv_heads=0)),
           (SHAPE, dict(n_heads=2048, n_kv_heads=1)), (INVALID, dict(max_pages=0)), (INVALID, dict(page_size=12)),
           (INVALID, dict(scale=float("inf"))), (INVALID, dict(scale=float("nan"))), (INVALID, dict(mask_words=0)),
           (SHAPE, dict(n_rows=2 ** 30, n_heads=8)), (INVALID, dict(q=P + 4)), (INVALID, dict(q_row_stride=1023)),
           (INVALID, dict(out_head_stride=12)), (INVALID, dict(k_token=255)), (INVALID, dict(v_page=1))]
    bad += [(INVALID, {n: None}) for n in ("q", "out", "k_data", "v_data", "block_table", "row_off", "ctx")]
    refuse("atspeed_tree_attention", bd.TreeAttentionArgs, ATTN, bad, P, 1 << 40)
    lib, n = bd.load_library(), C.c_size_t(0)
    assert lib.atspeed_tree_attention_workspace_bytes(C.byref(fill(bd.TreeAttentionArgs, **ATTN)), None) == INVALID
    assert lib.atspeed_tree_attention_workspace_bytes(C.byref(fill(bd.TreeAttentionArgs, **{**ATTN, "B": 0})), C.byref(n)) == INVALID
    for kw in (dict(n_rows=0), dict(max_new=0)):
        assert lib.atspeed_tree_attention(C.byref(fill(bd.TreeAttentionArgs, **{**ATTN, **kw})), None, 0, None) == OK


@pytest.mark.parametrize("kv_heads", [1, 3, 8, 511, 513, 1024])
@pytest.mark.parametrize("max_new", [1, 16, 40, 200])
def test_attention_workspace_of_long_contexts(kv_heads, max_new):
    """Parts of at most 2,048 workgroups of 128 queries (fp32 sums of 128 dims, two numbers a query)."""
    n = C.c_size_t(1)
    kw = dict(n_kv_heads=kv_heads, n_heads=kv_heads, max_pages=10 ** 6, max_ctx=10 ** 6, max_new=max_new, n_rows=400)
    assert bd.load_library().atspeed_tree_attention_workspace_bytes(C.byref(fill(bd.TreeAttentionArgs, **{**ATTN, **kw})), C.byref(n)) == OK
    assert n.value <= 2048 * 128 * (128 * 4 + 8) + 32
    # two requests: two pieces of each of their tiles
    assert (n.value > 0) == (kv_heads * 4 * -(-max_new // 128) <= 2048)


def test_rules_refusals():
    good = dict(dtype=bd.FP32, B=2, n_rows=5, n_cols=100, max_hist=10, max_nodes=4, mask_words=1, n_bias=2, n_states=3,
                n_out_rows=5, logits_stride=100, out_stride=100, bias_stride=100)
    bad = [(INVALID, dict(dtype=3)), (INVALID, dict(B=0)), (INVALID, dict(n_rows=-2)), (INVALID, dict(n_cols=0)),
           (INVALID, dict(n_cols=2 ** 20 + 1)), (INVALID, dict(logits=None)), (INVALID, dict(out=None)),
           (INVALID, dict(row_off=None)), (INVALID, dict(hist_len=None)), (INVALID, dict(history=None)),
           (INVALID, dict(max_hist=0)), (INVALID, dict(max_nodes=0)), (INVALID, dict(mask_words=0)),
           (INVALID, dict(n_bias=0)), (INVALID, dict(state=None)), (INVALID, dict(allowed=None)),
           (INVALID, dict(n_states=0)), (INVALID, dict(n_out_rows=0)), (SHAPE, dict(logits_stride=99)),
           (SHAPE, dict(out_stride=99)), (SHAPE, dict(bias_stride=99)), (INVALID, dict(logits=P, out=P)),
           (INVALID, dict(logits=P, out=P, out_row=None, out_stride=128)),
           (INVALID, dict(logits=P, out=P, out_row=None, dtype=bd.BF16))]
    refuse("atspeed_logit_rules", bd.LogitRulesArgs, good, bad)
    assert bd.load_library().atspeed_logit_rules(C.byref(fill(bd.LogitRulesArgs, **{**good, "n_rows": 0})), None) == OK


def test_rules_of_a_context_need_one():
    assert bd.load_library().atspeed_set_logit_rules(None, None) == INVALID


def test_tensors_that_are_not_on_a_gpu_are_refused():
    import torch
    from paper_2410_05165_amd import paged
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        paged.atspeed_page_plan(i(2), i(2), i(2), i(2, 3), i(5), i(1), 16, 4)
    c = torch.zeros(2, 16, 1, 64)
    with pytest.raises(ValueError):
        paged.atspeed_kv_append(c[0, :1], c[0, :1], c, c, i(1))
    with pytest.raises(ValueError):
        paged.atspeed_tree_attention(c[0, :1], c, c, i(1, 2), i(2), i(1), 5, 1)
    with pytest.raises(ValueError):
        paged.atspeed_logit_rules(torch.zeros(2, 5), i(2))

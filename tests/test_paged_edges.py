"""What needs the calls on PyTorch tensors (_marshal.so) and what does not, and calls past the largest launch (no
GPU needed)."""
import ctypes as C
import importlib
import os
import subprocess
import sys

import pytest

from paper_2410_05165_amd import binding as bd
from test_paged_args import ATTN, SHAPE, fill

build = importlib.import_module("paper_2410_05165_amd.build")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rules_of_a_context_do_without_the_tensor_calls():
    """Engine and its rules on a build of the library alone."""
    code = """
import sys
sys.modules["paper_2410_05165_amd._marshal"] = None          # not built
import torch
from paper_2410_05165_amd import binding
args = binding.pack_rules(32, 5, 2, torch.device("cuda:0"), mask_value=-3.0)
assert args.n_cols == 32 and args.token_base == 5 and args.B == 2 and args.mask_value == -3.0

class Lib:
    atspeed_set_logit_rules = staticmethod(lambda ctx, rules: 0)

eng = object.__new__(binding.Engine)
eng.lib, eng.ctx, eng.device, eng.torch, eng._rules = Lib, None, torch.device("cuda:0"), torch, {}
eng.w = type("W", (), dict(L=4, codebook=8, target=type("T", (), dict(item_base=5))))
eng.cfg = type("C", (), dict(max_batch=2))
eng.atspeed_set_logit_rules(mask_value=-3.0)
eng.atspeed_set_logit_rules()
try:
    import paper_2410_05165_amd.paged
except ImportError as e:
    assert "not built" in str(e)
else:
    raise AssertionError("the tensor calls did not miss their library")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_the_library_alone_is_built_by_hipcc_alone(monkeypatch):
    commands, moved = [], []
    monkeypatch.setattr(build, "_run", lambda cmd, verbose: commands.append(cmd))
    monkeypatch.setattr(build.os, "replace", lambda a, b: moved.append(b))
    assert build.build_library() == build.LIB
    assert {c[0] for c in commands} == {build.HIPCC} and len(commands) == len(build.SOURCES) + 1 and moved == [build.LIB]
    build.build()
    assert moved[1:] == [build.LIB, build.MARSHAL]


@pytest.mark.parametrize("n_rows,n_cols", [(2 ** 24, 1), (2 ** 24 + 5, 1024), (2 ** 18, 2 ** 18)])
def test_rules_past_the_largest_launch_are_refused(n_rows, n_cols):
    """A launch holds fewer than 2^32 threads, 2^24 workgroups of 256."""
    a = fill(bd.LogitRulesArgs, dtype=bd.FP32, B=2, n_rows=n_rows, n_cols=n_cols, max_hist=10, max_nodes=4, mask_words=1,
             n_bias=2, n_states=3, n_out_rows=5, logits_stride=n_cols, out_stride=n_cols, bias_stride=n_cols)
    assert bd.load_library().atspeed_logit_rules(C.byref(a), None) == SHAPE


@pytest.mark.parametrize("heads,rows", [(32, 2 ** 24), (8, 2 ** 25), (1, 2 ** 28)])
def test_appends_past_the_largest_launch_are_refused(heads, rows):
    a = fill(bd.KvAppendArgs, dtype=bd.BF16, n_rows=rows, n_kv_heads=heads, d_head=128, page_size=16, n_pool=10,
             k_row_stride=128 * heads, k_head_stride=128, v_row_stride=128 * heads, v_head_stride=128,
             k_page=2048 * heads, k_token=128 * heads, k_head=128, v_page=2048 * heads, v_token=128 * heads, v_head=128)
    assert bd.load_library().atspeed_kv_append(C.byref(a), None) == SHAPE


def test_attention_past_the_largest_launch_is_refused():
    """1,024 requests that are given no bound on their rows: 2,048 tiles of 128 queries for each and each of 8 heads."""
    kw = dict(B=1024, n_rows=65536, n_heads=32, n_kv_heads=8, max_new=65536, max_ctx=100, max_pages=5000)
    a, need = fill(bd.TreeAttentionArgs, **{**ATTN, **kw}), C.c_size_t(1)
    lib = bd.load_library()
    assert lib.atspeed_tree_attention_workspace_bytes(C.byref(a), C.byref(need)) == 0 and need.value == 0
    assert lib.atspeed_tree_attention(C.byref(a), None, 0, None) == SHAPE

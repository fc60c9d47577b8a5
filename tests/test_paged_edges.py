"""What needs the calls on PyTorch tensors (_marshal.so) and what does not (no GPU needed)."""
import importlib
import os
import subprocess
import sys

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
eng.lib, eng.ctx, eng.device, eng.stream = Lib, None, torch.device("cuda:0"), None
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

"""The native half of the scoring calls' binding: built for the installed torch, loaded by the first scoring call, and no
part of what compresses and restores."""
import os
import subprocess
import sys

import torch

from paper_2406_11257_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(code: str) -> str:
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stderr[-2000:]
    return out.stdout


def test_the_compressor_needs_no_scoring_binding():
    """As on a machine without a host compiler: the library loads, and only a scoring call fails, loudly."""
    assert "no compiler" in run("""
from paper_2406_11257_b200 import binding, build
def refuse(force=False):
    raise RuntimeError("no compiler")
build.build_binding = refuse
lib = binding.load_library()
assert binding.compress_bound(1000) > 0 and binding.mx4_bytes(8, 256, "e8m0_32") > 0
try:
    binding._score.mx4_quantize
except RuntimeError as e:
    print(e)
""")


def test_the_first_scoring_call_loads_it():
    assert "loaded" in run("""
from paper_2406_11257_b200 import binding
binding.load_library()
assert isinstance(binding._score, binding._NotLoaded)
assert callable(binding._score.mx4_linear) and callable(binding._score.token_logprobs)
assert not isinstance(binding._score, binding._NotLoaded) and binding.load_scoring() is binding._score
print("loaded")
""")


def test_another_torch_gets_another_file(monkeypatch):
    here = build.binding_path()
    assert os.path.dirname(here) == build.HERE and os.path.exists(build.build_binding())
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert build.binding_path() != here

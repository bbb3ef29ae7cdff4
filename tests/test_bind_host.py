"""The marshalling extension is tied to one Python and one torch: another one makes it stale, and without it everything but the 4-bit calls
works."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2510_04476_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

BLOCKED = """
import ctypes as C, sys
sys.modules["paper_2510_04476_b200._bind"] = None            # importing it raises ImportError
from paper_2510_04476_b200 import binding
lib = binding.load_library()
cfg = binding.cca_config(2048, 16, 4, 64, 2, 2, 2, 1, 63, 10000.0)
h = C.c_void_p()
assert lib.cca_init(C.byref(cfg), -1, C.byref(h)) == 0
n = C.c_size_t()
assert lib.cca_decode_workspace_size(h, 1, 128, C.byref(n)) == 0
lib.cca_destroy(h)
"""


def _run(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]


def test_another_torch_makes_the_extension_stale(monkeypatch):
    build.build()
    assert not build._stale()
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert build._stale()


def test_without_the_extension_the_library_still_loads():
    _run(BLOCKED + """
try:
    binding._BIND.qlinear(None)
except binding.CcaError as e:
    assert "_bind" in str(e)
else:
    raise AssertionError("a 4-bit call went through")
""")


@pytest.mark.gpu
def test_without_the_extension_the_bf16_path_runs():
    _run(BLOCKED + """
import torch
from paper_2510_04476_b200 import synth
sh = synth.Shape("bf16_alone", 1, 64, 256, 4, 2, 64)
w = {k: v.cuda() for k, v in synth.make_inputs(sh, want_dout=False).items() if v is not None}
cca = binding.CCA.from_shape(sh)
cca.forward(w, w["x"], cca.alloc_workspace(sh.B, sh.S, False))
torch.cuda.synchronize()
assert cca.last_status() == 0
try:
    cca.new_qcache(1, 8)
    cca.qlinear_pack(w["w_o"])
except binding.CcaError as e:
    assert "_bind" in str(e)
else:
    raise AssertionError("a 4-bit call went through")
cca.close()
""")

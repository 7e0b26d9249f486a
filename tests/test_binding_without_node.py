"""The ctypes binding needs the C library alone; the compiled module `_node` is asked for by the calls that it makes and by the modules."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MISSING = "sys.modules['paper_2510_27527_b200._node'] = None\n"
FOR_ANOTHER = "import types\nm = types.ModuleType('_node'); m.__file__ = 'there'; m.built_for = 'torch 1.0'\nsys.modules['paper_2510_27527_b200._node'] = m\n"


@pytest.mark.parametrize("state,message", [(MISSING, "_node"), (FOR_ANOTHER, "there is not for torch")])
def test_without_the_compiled_module(state, message):
    code = "import sys\nimport torch\n" + state + f"""
from paper_2510_27527_b200 import binding as b
assert b.lib.nvfp4_padded_k(100) == 128 and b.lib.nvfp4_ckpt8_ld(33) == 64
x = torch.zeros(1, 64, dtype=torch.bfloat16)
def modules():
    import paper_2510_27527_b200.module
def block():
    import paper_2510_27527_b200.block
for call in (lambda: b.nvfp4_ckpt8_pack(x), lambda: b.nvfp4_swiglu_fwd(x, x), modules, block):
    try:
        call()
    except ImportError as e:
        assert {message!r} in str(e) and "paper_2510_27527_b200.build" in str(e), str(e)
    else:
        raise AssertionError("not refused")
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert done.returncode == 0, done.stderr[-2000:]

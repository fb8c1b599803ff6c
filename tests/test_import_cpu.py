"""What importing the package brings with it."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(code):
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True, timeout=300)


def test_the_update_path_needs_no_torch():
    """The C ABI of the update path takes plain addresses; its binding loads where torch is not installed."""
    _run("""
import sys
sys.modules["torch"] = None                              # import torch raises ImportError
import paper_2504_18454_b200 as P
P.lib()
assert P.PREC_FP32 == 0 and P.strerror(-1) and callable(P.Palsgd)
try:
    P.ffn_forward
except ImportError:
    pass
else:
    raise AssertionError("the block operators need torch")
""")


def test_the_block_operators_are_there_when_asked_for():
    _run("""
import sys
import paper_2504_18454_b200 as P
assert "torch" not in sys.modules
assert {"ffn_forward", "Act8", "block", "Palsgd"} <= set(dir(P)) and not hasattr(P, "no_such_name")
assert "torch" not in sys.modules
assert P.ffn_forward is P.block.ffn_forward and P.SAVE_8BIT == 2 and "torch" in sys.modules
from paper_2504_18454_b200 import Act8, qk_norm_rope
names = {}
exec("from paper_2504_18454_b200 import *", names)
assert names["act8_pack"] is P.act8_pack and names["lib"] is P.lib and names["block"] is P.block
""")

"""The binding of the training-step operators without a GPU: what it needs to be imported, and what it refuses."""
import subprocess
import sys
from pathlib import Path

ROOT = Path(__file__).resolve().parent.parent

WITHOUT_TORCH = """
import sys
sys.modules["torch"] = None                                  # any import of it raises
from paper_2405_03637_b200 import binding as B
assert B.derive_scalars(B.make_hyper(1e-3, 0.9, 0.999, 1e-8, 0.0), 1)["b1"] == 0x3F66
assert B.workspace_bytes() > 0 and B.rms_norm_workspace_bytes(64) > 0
"""


def test_the_binding_does_without_torch_but_for_the_operators():
    p = subprocess.run([sys.executable, "-c", WITHOUT_TORCH], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert p.returncode == 0, p.stderr[-2000:]

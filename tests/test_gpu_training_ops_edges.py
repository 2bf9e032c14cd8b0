"""Training-step operators at the edges of their variants: sizes at which a launch changes its kind, several turns of
persistent kernels, zeros with a sign, values at the ends of the range."""
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent

# Rows whose slice takes between 43 and 49 KB of shared memory, each kernel's first launch of the process: the kernel's own
# 4.5 KB come on top of it, and beyond 48 KB in all a launch needs leave that an earlier, larger launch may have asked for.
FIRST_LAUNCHES = """
import torch
from paper_2405_03637_b200 import binding as B
for dtype, vocab in ((torch.bfloat16, 24_000), (torch.float32, 12_000)):
    rows, k = 300, 16
    z = torch.randn(rows, vocab, device="cuda").to(dtype)
    at, top = torch.arange(k, device="cuda").repeat(rows, 1), torch.zeros(rows, k, device="cuda")
    loss, dz = torch.empty(rows, device="cuda"), torch.empty_like(z)
    B.distill_loss_and_grad(z, at, top, 1.0, torch.ones(rows, device="cuda"), loss, dz)
    want = torch.logsumexp(z.double(), 1) - z[:, :k].double().mean(1) - torch.log(torch.tensor(float(k)))
    assert (loss.double() - want).abs().max() < 1e-4, vocab
"""


def test_first_launches_of_every_size_of_shared_memory():
    p = subprocess.run([sys.executable, "-c", FIRST_LAUNCHES], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr[-2000:]

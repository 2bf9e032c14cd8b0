"""The example that uses the training-step operators and the optimizer step together."""
import sys
from pathlib import Path

import pytest

sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width,ffn,vocab", [(256, 640, 4099), (136, 261, 1000)])
def test_the_student_learns_and_8_bits_follow(width, ffn, vocab):
    import distill_student
    curve, loss, loss8 = distill_student.run(steps=60, tokens=257, width=width, ffn=ffn, vocab=vocab)
    assert all(x == x for x in curve)
    assert sum(curve[-5:]) < 0.5 * sum(curve[:5]), curve              # it learns
    assert loss < 0.5 * curve[0]
    assert abs(loss8 - loss) < 0.05 * loss + 0.05                      # e4m3 operands: a few per cent of each activation

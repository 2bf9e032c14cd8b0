"""The example's training loop asks whether a kernel gave up one of its bounded waits."""
import sys
from pathlib import Path

import pytest

from paper_2405_03637_b200 import binding as B

sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))
pytestmark = pytest.mark.gpu


def test_a_wait_that_was_given_up_ends_the_training_with_an_error():
    import distill_student
    B.pipeline_fault()
    B.wait_timeout_selftest(5)                               # one warp waits 5 ms for nothing, leaves its code and returns
    with pytest.raises(RuntimeError, match="code 10[01]"):
        distill_student.run(steps=2, tokens=64, vocab=1000)
    assert B.pipeline_fault() == 0
    distill_student.run(steps=2, tokens=64, vocab=1000)

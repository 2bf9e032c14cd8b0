"""What the alignment example returns: the pairs' loss is a mean, and log 2 where the policy is its own reference."""
import math

import pytest

from test_gpu_align_example import example  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pairs", [1, 3, 8])
def test_the_first_loss_of_pairs_is_log_2(example, pairs):  # noqa: F811
    """Before its first step the policy has the reference's log-probabilities: every pair's loss is -log sigmoid(0), within a float's roundings of
    the weights, losses and their sum."""
    _, losses = example.run(steps=2, tokens=96, width=64, ffn=128, layers=1, vocab=301, pairs=pairs)
    assert len(losses) == 1 and abs(losses[0] - math.log(2)) < 16 * 2.0 ** -24

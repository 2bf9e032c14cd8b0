"""The preference loss's limit on the number of pairs, detected on the host before any CUDA call."""
import ctypes

from paper_2405_03637_b200 import binding as B
from test_alignment_ops_boundary_cpu import A


def test_pairs_are_below_2_to_the_30():
    """Each pair has two offsets, and arrays far apart (none of them is touched: without a device the next check ends the call)."""
    def call(pairs):
        far = lambda i: A + (i << 40)  # noqa: E731
        p = B.Preference(far(0), None, None, far(1), far(2), None, 8, 100, pairs, 8, 8, 0.1, 0.0, 0.0, 0)
        return B.lib().collage_preference_loss(ctypes.byref(p), None if pairs >= 1 << 30 else far(3) + 2, None, None, None)
    assert call(1 << 30) == B.ERR_LIMIT
    assert call((1 << 30) - 1) == B.ERR_ARG                               # past the limit's check: the loss is not aligned

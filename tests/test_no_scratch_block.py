"""The decoder block's kernels, which keep matrix accumulators in registers as the newer ones do,
use no scratch memory either."""
import pytest

from test_no_scratch import test_kernels_use_no_scratch_memory as check


@pytest.mark.parametrize("name", ["attend.hip", "cache.hip", "linear.hip", "norm.hip"])
def test_older_kernels_use_no_scratch_memory(name):
    check(name)

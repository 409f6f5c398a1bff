"""The GPU tests of the recurrence reach the plans that they are meant for: a rule that moves fails here,
without a GPU."""
import pytest

import layer_plans as plans


@pytest.mark.parametrize("shape,waves,split", plans.SCAN)
def test_recurrence(shape, waves, split):
    B, C, L = shape
    lanes, w, nseg = plans.scan_plan(B * C, L)
    assert (lanes, w, nseg > 1) == (64, waves, split)
    assert -(-L // 512) > w  # more than one turn of the wavefronts, or more than one segment

"""The example model: rows, recurrence, gradients and the optimiser together.

A candidate is of the history's topic or not, evenly: no model without the
history is better than log 2 = 0.693.  Served states differ from those read at
once by the rounding of fp32 recurrences of at most 60 steps over values below
some tens (bounded by 64 steps of 2^-20 each relative to them: 1e-2 is a
hundredfold room), and by nothing else: both read the same rounded rows."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("bits,dtype", [(32, "f32"), (32, "bf16"), (8, "bf16")])
def test_tower_learns_and_serves(bits, dtype):
    import sequence_tower
    losses, apart = sequence_tower.main(["--steps", "120", "--state-bits", str(bits), "--dtype", dtype])
    assert abs(losses[0] - 0.693) < 0.1
    assert sum(losses[-10:]) / 10 < 0.5
    assert apart < 1e-2

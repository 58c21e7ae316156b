"""The example's student acts in the simulator: the fused kernel's policy is the network that was taught."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_student_acts_by_the_fused_kernel():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import distill_policy
    finally:
        sys.path.pop(0)
    result = distill_policy.main(envs=1024, steps=32, epochs=6)
    # fp32 on both sides: two layers of 64 products each, and the inputs' scale taken into the
    # first layer's weights, a rounding each: 2^-24 (4 + 64 + 64) of sums of a few units
    assert result["apart"] < 1e-4
    assert abs(result["angle"] - result["teacher_angle"]) < 0.2 * result["teacher_angle"]

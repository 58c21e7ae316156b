"""The example runs: a student taught from a recorded rollout answers nearly as its teacher."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_distill_policy_example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import distill_policy
    finally:
        sys.path.pop(0)
    result = distill_policy.main()
    assert result["after"] < 0.2 * result["before"]
    assert result["same_draw"] > 0.95 and result["same_greedy"] > 0.9

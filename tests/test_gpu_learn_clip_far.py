"""Clipping by a factor below fp32's normal numbers: gradients near the largest numbers, and
limits near the smallest."""
import math

import pytest

torch = pytest.importorskip("torch")

import learn_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", (1000, 70000))          # one workgroup, many
@pytest.mark.parametrize("value,limit", [(1e38, 1.0), (3e38, 1e-6), (1e30, 1e-20), (1.0, 1e-38), (1e-3, 1e-41)])
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("own", (False, True))
def test_the_factor_keeps_its_digits(size, value, limit, dtype, own):
    import paper_2207_07736_amd as rl
    learner = rl.Learner()
    signs = torch.where(torch.arange(size, device="cuda") % 3 == 0, -1.0, 0.75)
    tensors = [(signs * value).to(dtype), (signs[:7] * (value * 2.0 ** -10)).to(dtype)]
    before = [t.double() for t in tensors]
    norm = math.sqrt(sum(float((t ** 2).sum()) for t in before))
    out = [torch.full_like(t, 5.0, dtype=torch.float32) for t in tensors] if own else tensors
    got = float(learner.clip(tensors, limit, out=out if own else None))
    learner.close()
    assert got == math.inf if norm > 3.5e38 else abs(got - norm) <= norm * (2.0 ** -24 + 2.0 ** -30)
    for b, t in zip(before, out):
        want = b * (limit / norm)
        # the factor's rounding and the product's; below the normal numbers a half step more for its place
        ref.close(t, want, ref.rounded(want, want.abs() * 2.5 * ref.U + 2.0 ** -149, t.dtype))

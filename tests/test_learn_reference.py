"""The learner's formulas (tests/learn_reference.py, 64 bits): their gradients against
differences of their values."""
import pytest

torch = pytest.importorskip("torch")

import learn_reference as ref  # noqa: E402


def _difference(f, args, k, direction, h=1e-6):
    """df along a direction of argument k, central."""
    value = []
    for sign in (1.0, -1.0):
        moved = list(args)
        moved[k] = args[k] + sign * h * direction
        value.append(float(f(*moved)))
    return (value[0] - value[1]) / (2 * h)


def _close(a, b):
    # the values are sums of some hundred terms of about 1: rounding moves a difference by 1e-14 / h
    # = 1e-8 for each of them, its second order by h^2
    assert abs(a - b) <= 1e-6 * max(1.0, abs(a)), (a, b)


@pytest.mark.parametrize("done", (False, True))
def test_recurrence(done):
    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    x, gate, state, dy, dlast = r(13, 3, 4), 2.0 * r(13, 3, 4), r(3, 4), r(13, 3, 4), r(3, 4)
    ends = (torch.rand((13, 3), generator=g) < 0.25) if done else None

    def total(x, gate, state):
        out = ref.scan(x, gate, state, ends)
        return (out[0][0] * dy).sum() + (out[1][0] * dlast).sum()

    _, _, dx, dgate, dstate = ref.scan(x, gate, state, ends, dy, dlast)
    for k, grad in enumerate((dx[0], dgate[0], dstate[0])):
        direction = r(*grad.shape)
        _close(_difference(total, (x, gate, state), k, direction), float((grad * direction).sum()))


def test_cross_entropy():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    hidden, matrix, weight = r(9, 5).float(), r(11, 5).float(), r(9).float()
    target = torch.randint(0, 11, (9,), generator=g)
    target[3], target[7], weight[5] = -1, 11, 0.0

    def total(hidden, matrix):
        z = hidden @ matrix.t()
        loss = torch.logsumexp(z, dim=1) - z.gather(1, target.clamp(0, 10)[:, None])[:, 0]
        return (torch.where((target >= 0) & (target < 11), loss, 0.0) * weight.double()).sum()

    (loss, _), (dx, _), (dw, _) = ref.xent(hidden, matrix, target, weight)
    _close(float((loss * weight.double()).sum()), float(total(hidden.double(), matrix.double())))
    for k, grad in enumerate((dx, dw)):
        direction = r(*grad.shape)
        _close(_difference(total, (hidden.double(), matrix.double()), k, direction), float((grad * direction).sum()))
    assert not dx[3].any() and not dx[7].any() and not dx[5].any()


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float16, torch.float32))
def test_bounds_are_small(dtype):
    """A bound that is not far above a rounding lets no other formula pass."""
    g = torch.Generator().manual_seed(2)
    hidden, matrix = torch.randn((20, 64), generator=g).to(dtype), (torch.randn((100, 64), generator=g) / 8).to(dtype)
    target = torch.randint(0, 100, (20,), generator=g)
    for value, err in ref.xent(hidden, matrix, target):
        # 32 bits: 100 terms of up to 70 u each in a sum, or a half step of 16 bits
        assert float(err.max()) <= (2e-4 if dtype == torch.float32 else 3.0 * ref.HALF_STEP[dtype]) * float(value.abs().max()) * 4
    x, gate = torch.randn((30, 2, 3), generator=g).to(dtype), torch.randn((30, 2, 3), generator=g).to(dtype)
    for value, err in ref.scan(x, gate, None, None, x):
        assert float(err.max()) <= 1e-4

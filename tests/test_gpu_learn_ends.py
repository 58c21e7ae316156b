"""What is not finite stays in its episode, whether the recurrence goes through time in one
piece or in segments that are joined.  The reference follows the definition: the end of an
episode takes 0 in place of the state, whatever the state is."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

# steps, sequences, channels; one piece below 64 steps or from 2 waves a CU on, else segments of
# 32 (48 for 5,003), which 16 runs of threads join, several segments to a run for the longer ones
SIZES = [(50, 3, 8), (64, 2, 4), (128, 3, 8), (200, 2, 7), (512, 2, 5), (5003, 1, 24), (4100, 3, 1), (96, 4096, 16)]
BAD = (float("nan"), float("inf"), -float("inf"))


@pytest.fixture(scope="module")
def learner():
    import paper_2207_07736_amd as rl
    made = rl.Learner()
    yield made
    made.close()


def _inputs(T, n, d, dtype, often):
    g = torch.Generator(device="cuda").manual_seed(T + d)
    x, dy = (torch.randn((T, n, d), generator=g, device="cuda").to(dtype) for _ in range(2))
    # gates of 0.02 to 0.5: products of a segment's gates go below the smallest number in some channels
    gate = torch.rand((T, n, d), generator=g, device="cuda") * 0.5 - 4.0 + 4.0 * torch.rand(d, generator=g, device="cuda")
    state, dlast = (torch.randn((n, d), generator=g, device="cuda") for _ in range(2))
    ends = (torch.rand((T, n), generator=g, device="cuda") < often).to(torch.uint8)
    for t in (31, 32, 40, 47, 63):                  # the last step of a segment, the first, and within
        if t < T:
            ends[t, t % n] = 3
    return x, gate.to(dtype), dy, state, dlast, ends


def _forward(bad, ends, state):
    """Which h_t, and which states that steps start from, are reached from `bad` steps."""
    hit, into, b = [], [], state.cpu()
    for t, end in zip(bad.cpu(), ends.cpu().bool()):
        into.append(b)
        hit.append(b | t)
        b = hit[-1] & ~end[:, None]
    return torch.stack(hit).cuda(), torch.stack(into).cuda(), b.cuda()


def _backward(bad, ends, dlast):
    """Which e_t are reached from `bad` gradients, and dstate."""
    hit, b = [], dlast.cpu()
    for t, end in zip(bad.cpu().flip(0), ends.cpu().bool().flip(0)):
        hit.append(t | (b & ~end[:, None]))
        b = hit[-1]
    return torch.stack(hit).flip(0).cuda(), b.cuda()


def _sites(T, n, d, seed):
    """One step in each channel of each sequence, at any place within its episodes."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    at = torch.randint(0, T, (n, d), generator=g, device="cuda")
    return torch.arange(T, device="cuda")[:, None, None] == at


def _same(value, hit):
    """value where hit, and nothing else that is not finite."""
    return lambda t: (torch.isnan(t) if math.isnan(value) else t == value) & hit | torch.isfinite(t) & ~hit


@pytest.mark.parametrize("often", (0.0, 1.0 / 60))
@pytest.mark.parametrize("value", BAD)
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16, torch.float16))
@pytest.mark.parametrize("T,n,d", SIZES)
def test_forward(learner, T, n, d, dtype, value, often):
    x, gate, _, state, _, ends = _inputs(T, n, d, dtype, often)
    clean = learner.scan(x, gate, state, ends, marks=True)
    for where in ("x", "state"):
        bad = _sites(T, n, d, 1) if where == "x" else torch.zeros((T, n, d), dtype=torch.bool, device="cuda")
        start = torch.zeros((n, d), dtype=torch.bool, device="cuda")
        rows, first = x.clone(), state.clone()
        rows[bad] = value
        if where == "state":
            start[:, ::2] = True
            first[start] = value
        hit, into, after = _forward(bad, ends, start)
        y, last, marks = learner.scan(rows, gate, first, ends, marks=True)
        for got, was, reached in ((y, clean[0], hit), (last, clean[1], after), (marks, clean[2], into[::16])):
            assert _same(value, reached)(got).all(), where
            assert torch.equal(got[~reached], was[~reached]), where


@pytest.mark.parametrize("often", (0.0, 1.0 / 60))
@pytest.mark.parametrize("value", BAD)
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16, torch.float16))
@pytest.mark.parametrize("T,n,d", SIZES)
def test_backward(learner, T, n, d, dtype, value, often):
    x, gate, dy, state, dlast, ends = _inputs(T, n, d, dtype, often)
    marks = learner.scan(x, gate, state, ends, marks=True)[2]
    clean = learner.scan_grad(x, gate, marks, dy, ends, dlast)
    for where in ("dy", "dlast"):
        bad = _sites(T, n, d, 2) if where == "dy" else torch.zeros((T, n, d), dtype=torch.bool, device="cuda")
        start = torch.zeros((n, d), dtype=torch.bool, device="cuda")
        rows, first = dy.clone(), dlast.clone()
        rows[bad] = value
        if where == "dlast":
            start[:, ::2] = True
            first[start] = value
        hit, before = _backward(bad, ends, start)
        dx, dgate, dstate = learner.scan_grad(x, gate, marks, rows, ends, first)
        assert _same(value, hit)(dx).all() and _same(value, before)(dstate).all(), where
        assert torch.equal(torch.isfinite(dgate), ~hit), where
        for got, was, reached in ((dx, clean[0], hit), (dgate, clean[1], hit), (dstate, clean[2], before)):
            assert torch.equal(got[~reached], was[~reached]), where


@pytest.mark.parametrize("value", BAD)
@pytest.mark.parametrize("T,n,d", SIZES)
def test_backward_of_rows_that_are_not_finite(learner, T, n, d, value):
    """x and the states it makes are factors of dgate alone."""
    x, gate, dy, state, dlast, ends = _inputs(T, n, d, torch.float32, 1.0 / 60)
    marks = learner.scan(x, gate, state, ends, marks=True)[2]
    clean = learner.scan_grad(x, gate, marks, dy, ends, dlast)
    bad, none = _sites(T, n, d, 3), torch.zeros((n, d), dtype=torch.bool, device="cuda")
    x[bad] = value
    marks = learner.scan(x, gate, state, ends, marks=True)[2]
    dx, dgate, dstate = learner.scan_grad(x, gate, marks, dy, ends, dlast)
    hit = _forward(bad, ends, none)[1] | bad
    assert torch.equal(dx, clean[0]) and torch.equal(dstate, clean[2])
    assert torch.equal(torch.isfinite(dgate), ~hit) and torch.equal(dgate[~hit], clean[1][~hit])


@pytest.mark.parametrize("T,n,d", SIZES)
def test_through_autograd(learner, T, n, d):
    """A NaN in one episode's rows reaches no other episode's gradients."""
    x, gate, dy, state, _, ends = _inputs(T, n, d, torch.float32, 1.0 / 60)
    bad, none = _sites(T, n, d, 4), torch.zeros((n, d), dtype=torch.bool, device="cuda")
    leaves = [t.clone().requires_grad_() for t in (x, gate, state)]
    with torch.no_grad():
        leaves[0][bad] = float("nan")
    h, last = learner.recur(*leaves, ends)
    hit, into, after = _forward(bad, ends, none)
    assert torch.equal(torch.isnan(h), hit) and torch.equal(torch.isnan(last), after)
    h.backward(dy)
    assert torch.isfinite(leaves[0].grad).all() and torch.isfinite(leaves[2].grad).all()
    assert torch.equal(torch.isnan(leaves[1].grad), into | bad)


def test_a_large_state_fades(learner):
    """Gates of 0.018 and no input: what a product below the smallest number carries of a finite
    state is nothing, not the smallest number's share."""
    T, n, d = 512, 2, 5
    x, gate = torch.zeros((T, n, d), device="cuda"), torch.full((T, n, d), -4.0, device="cuda")
    state = torch.full((n, d), 1e30, device="cuda")
    y, last = learner.scan(x, gate, state)
    t = torch.arange(1, T + 1, device="cuda", dtype=torch.float64)[:, None, None]
    # each gate is off by 16 units of 2^-24 at most
    most = state.double() * torch.exp(t * (math.log(1.0 / (1.0 + math.exp(4.0))) + 2.0 ** -19)) + 2.0 ** -149
    assert (y >= 0).all() and (y.double() <= most).all() and not last.any()
    dy = torch.zeros_like(x)
    marks = learner.scan(x, gate, state, marks=True)[2]
    dx, _, dstate = learner.scan_grad(x, gate, marks, dy, None, state)
    assert (dx >= 0).all() and (dx.double() <= most.flip(0) * 57.0).all() and not dstate.any()

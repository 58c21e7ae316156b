"""The learner's operators one after the other, as a training step on a recorded rollout uses
them: against the formulas, through autograd, in captured graphs, on other streams."""
import math

import pytest

torch = pytest.importorskip("torch")

import learn_reference as ref  # noqa: E402
import workloads  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rollout():
    """Rows of 120 steps of 300 cart-poles: features of the observations, actions, ends of
    episodes, and an advantage for each step."""
    from paper_2207_07736_amd import Simulator, Trajectory
    sim = Simulator(300, 0, workloads.CARTPOLE)
    sim.reset(5)
    tr = Trajectory(120, sim.n)
    sim.step(120, tr.rows(0, 120))
    torch.cuda.synchronize()
    g = torch.Generator(device="cuda").manual_seed(0)
    obs = tr.learner_batch()["obs"].contiguous()
    first = torch.randn((4, 48), generator=g, device="cuda")
    x, gate = obs @ first, obs @ torch.randn((4, 48), generator=g, device="cuda") + 1.0
    advantage = torch.randn(120 * 300, generator=g, device="cuda")
    sim.close()
    return x, gate, tr.action, tr.done, advantage


def _step(learner, x, gate, state, done, matrix, action, weight, out=None):
    """One training step's calls; returns all that it makes."""
    y, last, marks = learner.scan(x, gate, state, done, marks=True)
    loss, dhidden, dmatrix = learner.cross_entropy(y.view(-1, x.shape[2]), matrix, action, weight)
    dx, dgate, dstate = learner.scan_grad(x, gate, marks, dhidden.view_as(y), done)
    norm = learner.clip([dx, dgate, dmatrix], 1.0, out=out)
    return y, last, loss, dhidden, dmatrix, dx, dgate, dstate, norm


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16, torch.float16))
def test_a_training_step(rollout, dtype):
    import paper_2207_07736_amd as rl
    x, gate, action, done, weight = rollout
    x, gate = x.to(dtype), gate.to(dtype)
    assert done.any() and int(action.max()) == 1
    matrix = (torch.randn((5, 48), device="cuda") / 7).to(dtype)
    state = torch.zeros((300, 48), device="cuda")
    learner = rl.Learner(120 * 300, 48, 5)
    try:
        out = [torch.empty_like(x, dtype=torch.float32), torch.empty_like(x, dtype=torch.float32),
               torch.empty_like(matrix, dtype=torch.float32)]
        y, last, loss, dhidden, dmatrix, dx, dgate, dstate, norm = _step(learner, x, gate, state, done, matrix, action.view(-1), weight, out)
        h, l, *_ = ref.scan(x, gate, state, done)
        ref.close(y, h[0], ref.rounded(*h, dtype), "y")
        ref.close(last, *l, "last")
        want = ref.xent(y.view(-1, 48), matrix, action.view(-1), weight)
        ref.close(loss, want[0][0], want[0][1] + want[0][0].abs() * ref.U, "loss")
        ref.close(dhidden, want[1][0], ref.rounded(*want[1], dtype), "dhidden")
        ref.close(dmatrix, want[2][0], ref.rounded(*want[2], dtype), "dmatrix")
        _, _, gx, gg, gs = ref.scan(x, gate, state, done, dhidden.view_as(y))
        ref.close(dx, gx[0], ref.rounded(*gx, dtype), "dx")
        ref.close(dgate, gg[0], ref.rounded(*gg, dtype), "dgate")
        ref.close(dstate, *gs, "dstate")
        total = math.sqrt(sum(float((t.double() ** 2).sum()) for t in (dx, dgate, dmatrix)))
        assert total > 1.0 and abs(float(norm) - total) <= total * (ref.U + 2.0 ** -30)
        for o, t in zip(out, (dx, dgate, dmatrix)):
            ref.close(o, t.double() / total, ref.rounded(t.double() / total, t.double().abs() / total * 2.5 * ref.U, torch.float32))

        # through autograd: the same bits
        leaves = [t.clone().requires_grad_() for t in (x, gate, matrix, state)]
        ay, alast = learner.recur(leaves[0], leaves[1], leaves[3], done)
        (learner.cross_entropy_loss(ay.reshape(-1, 48), leaves[2], action.view(-1)) * weight).sum().backward()
        assert torch.equal(ay, y) and torch.equal(alast, last)
        for leaf, grad in zip(leaves, (dx, dgate, dmatrix, dstate)):
            assert torch.equal(leaf.grad, grad)
        # and clipped in place, as an optimiser's parameters
        assert torch.equal(learner.clip([p.grad for p in leaves[:3]], 1.0), norm)
        for leaf, o in zip(leaves, out):
            ref.close(leaf.grad, o.double(), ref.rounded(o.double(), o.double().abs() * ref.U, dtype))
    finally:
        learner.close()


def test_a_broadcast_gradient_and_a_shared_leaf():
    """y.sum() hands autograd an expanded gradient; x that is its own gate gets both."""
    import paper_2207_07736_amd as rl
    learner = rl.Learner()
    x = torch.randn((40, 3, 10), device="cuda", requires_grad=True)
    y, last = learner.recur(x, x)
    y.sum().backward()
    _, _, gx, gg, _ = ref.scan(x.detach(), x.detach(), None, None, torch.ones_like(x))
    ref.close(x.grad, gx[0] + gg[0], ref.rounded(gx[0] + gg[0], ref.rounded(*gx, torch.float32) + ref.rounded(*gg, torch.float32), torch.float32))
    x.grad = None
    learner.recur(x, x)[1].sum().backward()                # the last state alone
    _, _, gx, gg, _ = ref.scan(x.detach(), x.detach(), None, None, None, torch.ones((3, 10), device="cuda"))
    ref.close(x.grad, gx[0] + gg[0], ref.rounded(gx[0] + gg[0], ref.rounded(*gx, torch.float32) + ref.rounded(*gg, torch.float32), torch.float32))
    learner.close()


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16, torch.float16))
@pytest.mark.parametrize("T,n,d,V", [(1, 8, 32, 20), (500, 2, 64, 700), (64, 40, 200, 3000)])
def test_a_captured_step_replays(T, n, d, V, dtype):
    """Replays with eager calls, other tensors' work and synchronizations between."""
    import paper_2207_07736_amd as rl
    stream = torch.cuda.Stream()
    learner, other = rl.Learner(T * n, d, V, stream=stream), rl.Learner(T * n, d, V, stream=stream)
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, gate, matrix, state, weight = r(T, n, d).to(dtype), r(T, n, d).to(dtype), (r(V, d) / 8).to(dtype), r(n, d), r(T * n)
    done = (torch.rand((T, n), generator=g, device="cuda") < 0.05).to(torch.uint8)
    action = torch.randint(-1, V, (T * n,), generator=g, device="cuda", dtype=torch.int32)
    out = [torch.empty_like(x), torch.empty_like(x), torch.empty_like(matrix)]
    args = (x, gate, state, done, matrix, action, weight, out)
    torch.cuda.synchronize()
    try:
        with torch.cuda.stream(stream):
            _step(learner, *args)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                made = _step(learner, *args)
            for turn in range(4):
                x.copy_(r(T, n, d))                        # other rows each time
                state.copy_(r(n, d))
                torch.cuda.synchronize()
                want = [t.clone() for t in _step(other, *args)] + [o.clone() for o in out]
                torch.cuda.synchronize()
                for t in (*made, *out):
                    t.zero_()
                learner.clip([torch.ones(100000, device="cuda")], 5.0)          # eager work in the same workspace
                stream.synchronize()
                graph.replay()
                stream.synchronize()
                for k, (a, b) in enumerate(zip((*made, *out), want)):
                    assert torch.equal(a, b), (turn, k)
            del graph, made
    finally:
        learner.close()
        other.close()


@pytest.mark.parametrize("current_own", (False, True))
@pytest.mark.parametrize("handle_own", (False, True))
def test_gradients_off_the_handles_stream(handle_own, current_own):
    import paper_2207_07736_amd as rl
    handle = torch.cuda.Stream() if handle_own else None
    current = torch.cuda.Stream() if current_own else torch.cuda.default_stream()
    learner, plain = rl.Learner(600, 64, 3000, stream=handle), rl.Learner(600, 64, 3000)
    busy = torch.zeros((4096, 4096), device="cuda", dtype=torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(3)
    try:
        for T, n in ((300, 2), (4, 100)):
            for turn in range(3):
                x, matrix = torch.randn((T, n, 64), generator=g, device="cuda"), torch.randn((3000, 64), generator=g, device="cuda")
                target = torch.randint(0, 3000, (T * n,), generator=g, device="cuda")
                y, _, marks = plain.scan(2.0 * x, x, marks=True)
                loss, dh, dm = plain.cross_entropy(y.view(-1, 64), matrix, target)
                dx, dg, _ = plain.scan_grad(2.0 * x, x, marks, dh.view_as(y))
                torch.cuda.synchronize()
                with torch.cuda.stream(current):
                    leaf, gates, mat = (t.clone().requires_grad_() for t in (x, x, matrix))
                    for _ in range(12):                      # a millisecond of work ahead of the rows
                        busy = busy @ busy
                    rows = leaf * (2.0 + busy[0, 0].float())
                    h, _ = learner.recur(rows, gates)
                    losses = learner.cross_entropy_loss(h.reshape(-1, 64), mat, target)
                    kept = losses.detach().clone()
                    for _ in range(12):                      # and of the losses' gradient
                        busy = busy @ busy
                    (losses * (1.0 + busy[0, 0].float())).sum().backward()
                    grads = [t.grad.clone() for t in (leaf, gates, mat)]
                    del losses, h, rows, leaf, gates, mat
                    torch.full((3000, 64), float("nan"), device="cuda")          # over whatever was freed
                torch.cuda.synchronize()
                for a, b in zip((kept, *grads), (loss, dx * 2.0, dg, dm)):
                    assert torch.equal(a, b), (T, n, turn)
    finally:
        learner.close()
        plain.close()


def test_two_learners_side_by_side():
    import paper_2207_07736_amd as rl
    streams = [torch.cuda.Stream() for _ in range(2)]
    learners = [rl.Learner(500, 256, 5000, stream=s) for s in streams]
    g = torch.Generator(device="cuda").manual_seed(4)
    hidden = torch.randn((500, 256), generator=g, device="cuda").bfloat16()
    matrix = (torch.randn((5000, 256), generator=g, device="cuda") / 16).bfloat16()
    target = torch.randint(0, 5000, (500,), generator=g, device="cuda")
    long = torch.randn((4000, 1, 64), generator=g, device="cuda")
    torch.cuda.synchronize()
    want = None
    for turn in range(3):
        made = []
        for learner, s in zip(learners, streams):
            with torch.cuda.stream(s):
                y, last = learner.scan(long, long)
                made.append((*learner.cross_entropy(hidden, matrix, target), y, last, learner.clip([long], math.inf)))
        torch.cuda.synchronize()
        want = want or [t.clone() for t in made[0]]
        for parts in made:
            for a, b in zip(parts, want):
                assert torch.equal(a, b), turn
    for learner in learners:
        learner.close()


def test_closed_and_empty():
    import paper_2207_07736_amd as rl
    learner = rl.Learner()
    learner.close()
    learner.close()
    x = torch.zeros((2, 1, 4), device="cuda")
    with pytest.raises(rl.RlsimError):
        learner.scan(x, x)
    with pytest.raises(rl.RlsimError, match="all 0 or none"):
        rl.Learner(5, 0, 7)

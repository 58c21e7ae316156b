"""examples/recurrent_policy.py runs, and its gradients are those of the same model in torch."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import recurrent_policy
        yield recurrent_policy
    finally:
        sys.path.remove(os.path.join(ROOT, "examples"))


def test_it_runs(example):
    result = example.main(envs=256, steps=40, epochs=3)
    assert torch.isfinite(result["losses"]).all() and (result["norms"] > 0).all()
    assert result["answers"].shape == (40, 256) and set(result["answers"].unique().tolist()) <= {0, 1}
    total = sum(float((g.double() ** 2).sum()) for g in result["gradients"]) ** 0.5
    assert total <= min(0.5, float(result["norms"][-1])) * (1 + 1e-5)      # clipped


def test_its_gradients(example):
    """Against autograd through the formulas in 64 bits.  A gradient sums 1,920 rows' terms, each
    from sums of 32 and 30 steps of some four roundings: 2,072 roundings of 2^-24 that add up
    like random ones, 2.7e-6 of the terms' absolute sum.  Terms of either sign leave 1/44 (the
    root of 1,920) of that sum: 1.2e-4 of the gradient; 1e-3 allows eight times it."""
    import paper_2207_07736_amd as rl
    obs, action, reward, done = example.rollout(64, 30, seed=3)
    weight = example.returns(reward, done).reshape(-1)
    torch.manual_seed(1)
    learner = rl.Learner(30 * 64, 32, 2)
    policy = example.Policy(learner).cuda()
    rows, _ = policy(obs, done)
    (learner.cross_entropy_loss(rows.reshape(-1, 32), policy.output, action.reshape(-1)) * weight).mean().backward()
    got = [p.grad.clone() for p in policy.parameters()]

    twin = example.Policy(None).cuda().double()
    twin.load_state_dict({k: v.double() for k, v in policy.state_dict().items()})
    x, a = twin.input(obs.double()), torch.sigmoid(twin.gate(obs.double()))
    h, out = torch.zeros((64, 32), dtype=torch.float64, device="cuda"), []
    for t in range(30):
        h = a[t] * h + (1 - a[t]) * x[t]
        out.append(h)
        h = h * (done[t] == 0)[:, None]
    z = torch.stack(out).reshape(-1, 32) @ twin.output.t()
    loss = torch.logsumexp(z, dim=1) - z.gather(1, action.reshape(-1, 1).long())[:, 0]
    (loss * weight.double()).mean().backward()
    for g, p in zip(got, twin.parameters()):
        assert float((g.double() - p.grad).norm()) <= 1e-3 * float(p.grad.norm())
    learner.close()

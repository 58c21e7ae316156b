"""Train a recurrent policy on a recorded rollout with the learner's operators.

1. The simulator steps cart-pole environments and records observations, the random actions
   taken and where episodes end (rlsim_step_fused).
2. A recurrent core (two torch layers for its input and its gate, Learner.recur over the
   recorded steps, reset where episodes end) and an output layer over the actions learn to
   raise the probability of the actions of steps with a high return: each step's
   cross entropy (Learner.cross_entropy_loss) weighs by its discounted return, normalised.
3. Gradients are clipped by their global norm (Learner.clip) before the optimiser's step.
4. The policy acts: one step of the recurrence at a time (Learner.scan of one step), its
   actions drawn by Head.sample.  The simulators draw their actions themselves, so these are
   for rows recorded before.

    python examples/recurrent_policy.py [--envs 1024] [--steps 64] [--epochs 6]
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2207_07736_amd as rl  # noqa: E402
import workloads  # noqa: E402


def rollout(envs, steps, seed):
    """Observations [steps, envs, 4], actions, rewards and ends of episodes [steps, envs]."""
    sim = rl.Simulator(envs, 0, workloads.CARTPOLE)
    try:
        sim.reset(seed)
        traj = rl.Trajectory(steps, envs)
        sim.step(steps, traj.rows(0, steps))
        batch = traj.learner_batch()
        return batch["obs"].contiguous(), traj.action, traj.reward, traj.done
    finally:
        sim.close()


def returns(reward, done, discount=0.97):
    """Discounted returns within the episodes, over their mean and deviation."""
    out = torch.empty_like(reward)
    ahead = torch.zeros_like(reward[0])
    for t in reversed(range(reward.shape[0])):
        ahead = reward[t] + discount * ahead * (done[t] == 0)
        out[t] = ahead
    return (out - out.mean()) / out.std()


class Policy(torch.nn.Module):
    def __init__(self, learner, width=32, actions=2):
        super().__init__()
        self.learner = learner
        self.input, self.gate = torch.nn.Linear(4, width), torch.nn.Linear(4, width)
        self.output = torch.nn.Parameter(torch.randn(actions, width) / width ** 0.5)

    def forward(self, obs, done):
        """The recurrence's rows [steps, envs, width] and its last state."""
        return self.learner.recur(self.input(obs), self.gate(obs), None, done)


def main(envs=1024, steps=64, epochs=6):
    torch.manual_seed(0)
    obs, action, reward, done = rollout(envs, steps, seed=0)
    weight = returns(reward, done).reshape(-1)
    learner = rl.Learner(steps * envs, 32, 2)
    policy = Policy(learner).cuda()
    optimiser = torch.optim.Adam(policy.parameters(), lr=3e-3)
    losses, norms = [], []
    for _ in range(epochs):
        rows, _ = policy(obs, done)
        loss = learner.cross_entropy_loss(rows.reshape(-1, 32), policy.output, action.reshape(-1))
        total = (loss * weight).mean()
        optimiser.zero_grad()
        total.backward()
        norms.append(learner.clip([p.grad for p in policy.parameters()], 0.5))
        optimiser.step()
        losses.append(total.detach())

    head = rl.Head(envs, 2)
    state, answers = torch.zeros((envs, 32), device="cuda"), []
    with torch.no_grad():
        for t in range(steps):
            h, state = learner.scan(policy.input(obs[t])[None], policy.gate(obs[t])[None], state, done[t:t + 1], last=state)
            answers.append(head.sample(h[0] @ policy.output.t(), torch.rand(envs, device="cuda")))
    torch.cuda.synchronize()
    result = dict(losses=torch.stack(losses).cpu(), norms=torch.stack(norms).cpu(), answers=torch.stack(answers).cpu(),
                  gradients=[p.grad.detach().cpu() for p in policy.parameters()])
    head.close()
    learner.close()
    return result


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    for name, value in (("envs", 1024), ("steps", 64), ("epochs", 6)):
        parser.add_argument("--" + name, type=int, default=value)
    out = main(**vars(parser.parse_args()))
    print("weighted losses", [round(float(v), 4) for v in out["losses"]])
    print("gradient norms before clipping", [round(float(v), 4) for v in out["norms"]])
    print("share of action 1 drawn", float(out["answers"].float().mean()))

"""Teach a student what the fused MLP policy answers, then let it answer and act itself.

1. The fused kernel steps cart-pole environments with the MLP policy and records each
   step's observation and the policy's probability of action 0 (rlsim_step_fused).
2. A student network in torch, of the fused policy's shape, learns from the recorded
   rows: each row's teacher gives its top logits, here both actions' log probabilities,
   and Head.distill_loss is the loss it trains on.
3. On the rows of a fresh rollout the student answers by Head.sample, with uniform
   numbers of one's own, greedily and at temperature 1.  The simulators draw their actions
   themselves and take none from outside, so these answers are for comparison.
4. The student acts: its weights are the fused kernel's policy for a rollout of its own.

    python examples/distill_policy.py [--envs 4096] [--steps 64] [--epochs 8]
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


def teacher_policy():
    """The policy workload's weights on the device, scaled to give decided answers."""
    w = {key: torch.from_numpy(value).cuda() for key, value in workloads.mlp_weights(0).items()}
    w["w1"], w["w3"] = w["w1"] * 4.0, w["w3"] * 4.0
    keep = [w[key].contiguous() for key in ("w1", "b1", "w2", "b2", "w3", "b3")]
    return rl.policy_struct(rl.RLSIM_F32, *keep), keep


def rollout(policy, envs, steps, seed):
    """Observations [steps * envs, 4] and the policy's p0 [steps * envs]."""
    sim = rl.Simulator(envs, 0, workloads.CARTPOLE)
    try:
        sim.reset(seed)
        traj = rl.Trajectory(steps, envs, p0=True)
        sim.step(steps, traj.rows(0, steps), policy)
        obs = traj.learner_batch()["obs"].reshape(-1, 4).contiguous()
        return obs, traj.policy_p0.reshape(-1).clone()
    finally:
        sim.close()


def student_policy(net, spread):
    """The network as rlsim_step_fused takes it, its scaled inputs folded into the first layer."""
    first, _, second, _, last = net
    keep = [(first.weight / spread).detach().contiguous()]
    keep += [v.detach().contiguous() for v in (first.bias, second.weight, second.bias, last.weight, last.bias)]
    return rl.policy_struct(rl.RLSIM_F32, *keep), keep


def main(envs=4096, steps=64, epochs=8, batch=8192):
    torch.manual_seed(0)
    policy, keep = teacher_policy()
    obs, p0 = rollout(policy, envs, steps, seed=1)
    logits_t = torch.stack((torch.log(p0), torch.log1p(-p0)), dim=1)
    index = torch.arange(2, dtype=torch.int32, device="cuda").expand(len(p0), 2).contiguous()
    net = torch.nn.Sequential(torch.nn.Linear(4, 64), torch.nn.Tanh(), torch.nn.Linear(64, 64), torch.nn.Tanh(),
                              torch.nn.Linear(64, 2)).cuda()
    spread = obs.std(dim=0)                       # the four words differ in scale by ten

    def student(o):
        return net(o / spread)

    optimizer = torch.optim.Adam(net.parameters(), lr=5e-3)
    fresh, fresh_p0 = rollout(policy, envs, steps, seed=2)
    head = rl.Head(max(batch, len(fresh)), 2)
    try:
        def divergence(o, p):
            t = torch.stack((torch.log(p), torch.log1p(-p)), dim=1)
            return head.distill(student(o).detach(), t, index[:len(p)], grad=False).mean().item()

        before = divergence(fresh, fresh_p0)
        for _ in range(epochs):
            for rows in torch.randperm(len(obs), device="cuda").split(batch):
                loss = head.distill_loss(student(obs[rows]), logits_t[rows], index[rows]).mean()
                optimizer.zero_grad()
                loss.backward()
                optimizer.step()
        after = divergence(fresh, fresh_p0)
        u = torch.rand(len(fresh), device="cuda")
        answer = student(fresh).detach()
        action, logp = head.sample(answer, u, logp=True)
        greedy = head.sample(answer, u, temperature=0.0)
        same_draw = (action == (u >= fresh_p0).int()).float().mean().item()     # the teacher's draw from the same numbers
        same_greedy = (greedy == (fresh_p0 < 0.5).int()).float().mean().item()
        policy, keep = student_policy(net, spread)
        own, own_p0 = rollout(policy, envs, steps, seed=2)
        # what the fused kernel acted by, on the rows that it met
        apart = (own_p0 - torch.softmax(student(own).detach(), dim=1)[:, 0]).abs().max().item()
        torch.cuda.synchronize()
    finally:
        head.close()
    print(f"KL(teacher || student) on a fresh rollout: {before:.4f} before, {after:.5f} after {epochs} epochs")
    print(f"same action as the teacher: {same_draw:.4f} drawn, {same_greedy:.4f} greedy; mean log-probability {logp.mean().item():.4f}")
    print(f"acting itself from the same start: mean |pole angle| {own[:, 2].abs().mean().item():.5f}, the teacher's "
          f"{fresh[:, 2].abs().mean().item():.5f}; p0 of the fused kernel within {apart:.1e} of the network's")
    return dict(apart=apart, angle=own[:, 2].abs().mean().item(), teacher_angle=fresh[:, 2].abs().mean().item(), before=before, after=after, same_draw=same_draw, same_greedy=same_greedy)


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    parser.add_argument("--envs", type=int, default=4096)
    parser.add_argument("--steps", type=int, default=64)
    parser.add_argument("--epochs", type=int, default=8)
    args = parser.parse_args()
    main(args.envs, args.steps, args.epochs)

"""A policy with memory on the simulator: acts one step at a time, learns from whole rollouts.

    python examples/policy_memory.py [--envs N] [--steps T] [--updates U] [--dtype bf16|f32]

Two recurrent blocks (short causal convolution, selective state space scan, and the norm that joins a
block to the next) between an embedding of Craftax-Classic's symbolic observation and the heads for
actions and values.  While acting, the blocks take one token per environment and carry their states;
an environment whose episode has ended starts with empty ones, by the simulator's own `done`.  For
the update the same blocks take the rollout as [steps][n] sequences, from the states it began with,
and give the gradients of an advantage actor-critic loss.  Per update it prints the mean reward, the loss and
how far the logits of the two forms are apart.  Weights are float32 and are rounded to the type of
the activations where they are used.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2402_16801_amd import binding as cx, memory, synth  # noqa: E402

ACTIONS = 17


def times(v, weight):
    return v @ weight.to(v.dtype)


class Block(torch.nn.Module):
    def __init__(self, width, inner=None, states=16, taps=4, rank=16, dtype=torch.bfloat16):
        super().__init__()
        inner = 2 * width if inner is None else inner

        def weight(rows, columns):
            return torch.nn.Parameter(torch.randn(rows, columns, device="cuda") * rows ** -0.5)

        def vector(value, size):
            return torch.nn.Parameter(torch.full((size,), value, device="cuda"))

        self.inner, self.states, self.rank, self.taps, self.dtype = inner, states, rank, taps, dtype
        self.w_in, self.w_out = weight(width, 2 * inner), weight(inner, width)
        self.w_scan, self.w_delta = weight(inner, rank + 2 * states), weight(rank, inner)
        self.conv_weight = torch.nn.Parameter(torch.randn(inner, taps, device="cuda") * taps ** -0.5)
        self.conv_bias = vector(0.0, inner)
        # rates -1 .. -states, steps of about 0.01: memories from ten to some hundred steps
        self.log_a = torch.nn.Parameter(torch.arange(1.0, states + 1, device="cuda").log().repeat(inner, 1))
        self.delta_bias, self.d = vector(-4.6, inner), vector(1.0, inner)
        self.post_weight, self.scale, self.pre_weight = vector(1.0, width), vector(0.5, width), vector(1.0, width)

    def empty(self, n):
        return [torch.zeros(n, self.taps - 1, self.inner, dtype=self.dtype, device="cuda"),
                torch.zeros(n, self.inner, self.states, device="cuda")]

    def forward(self, residual, u, state, first):
        """(residual, u, state) after the block.  [n][width] is one step, its state updated in place;
        [steps][n][width] a rollout from the given state."""
        step = u.dim() == 2
        x, z = times(u, self.w_in).split(self.inner, -1)
        if step:
            x, _ = memory.causal_conv_step(x, self.conv_weight, self.conv_bias, state[0], first=first)
        else:
            x, tail = memory.conv(x, self.conv_weight, self.conv_bias, state=state[0], first=first)
        rank, b, c = times(x, self.w_scan).split([self.rank, self.states, self.states], -1)
        delta, b, c, a = times(rank, self.w_delta), b.unsqueeze(-2), c.unsqueeze(-2), -self.log_a.exp()
        how = {"d": self.d, "z": z, "delta_bias": self.delta_bias, "first": first}
        if step:
            y, _ = memory.selective_scan_step(x, delta, a, b, c, state[1], **how)
        else:
            y, h = memory.scan(x, delta, a, b, c, state=state[1], **how)
            state = [tail, h]
        norms = {"post_weight": self.post_weight, "scale": self.scale, "pre_weight": self.pre_weight}
        y = times(y, self.w_out)
        if step:        # one token as a sequence of one step
            residual, u = (v[0] for v in memory.residual_norm(y[None], residual[None], **norms))
        else:
            residual, u = memory.norm(y, residual, **norms)
        return residual, u, state


class Policy(torch.nn.Module):
    def __init__(self, inputs, width=256, blocks=2, dtype=torch.bfloat16, **how):
        super().__init__()
        self.dtype = dtype
        self.embed = torch.nn.Parameter(torch.randn(inputs, width, device="cuda") * inputs ** -0.5)
        self.blocks = torch.nn.ModuleList(Block(width, dtype=dtype, **how) for _ in range(blocks))
        self.head = torch.nn.Parameter(torch.randn(width, ACTIONS + 1, device="cuda") * (0.1 * width ** -0.5))

    def empty(self, n):
        return [block.empty(n) for block in self.blocks]

    def forward(self, obs, states, first):
        """(logits, values, states)"""
        residual = u = times(obs.to(self.dtype), self.embed)
        after = []
        for block, state in zip(self.blocks, states):
            residual, u, state = block(residual, u, state, first)
            after.append(state)
        out = times(u, self.head).float()
        return out[..., :ACTIONS], out[..., ACTIONS], after


@torch.no_grad()
def act(policy, sim, states, first, steps):
    """Plays `steps` steps: what was seen, done and earned, [steps][n] each, and `ahead`, the value of what is seen behind the last
    step, [n].  states and first are carried on in place."""
    n, seen = sim.n, {k: [] for k in ("obs", "first", "logits", "actions", "reward", "done")}
    for _ in range(steps):
        obs = sim.obs.view(torch.float32)
        logits, _, _ = policy(obs, states, first)
        actions = (logits - torch.empty_like(logits).exponential_().log()).argmax(-1).to(torch.int32)      # a draw from softmax(logits)
        for k, v in (("obs", obs), ("first", first), ("logits", logits), ("actions", actions)):
            seen[k].append(v.clone())
        _, reward, done = sim.step(actions)
        seen["reward"].append(reward.clone())
        seen["done"].append(done.clone())
        first.copy_(done)
    seen = {k: torch.stack(v) for k, v in seen.items()}
    _, seen["ahead"], _ = policy(sim.obs.view(torch.float32), [[v.clone() for v in state] for state in states], first)
    return seen


def loss_of(policy, seen, states, discount=0.99):
    """(actor-critic loss over a rollout that began with `states`, logits).  The return of the last step goes on with the value of what
    followed it, as acting saw it."""
    logits, values, _ = policy(seen["obs"], states, seen["first"])
    with torch.no_grad():
        returns, ahead = torch.empty_like(values), seen["ahead"].to(values.dtype)
        for t in range(len(values) - 1, -1, -1):
            ahead = returns[t] = seen["reward"][t] + discount * ahead * (1 - seen["done"][t].float())
        advantage = returns - values
    chosen = torch.distributions.Categorical(logits=logits, validate_args=False)
    actor = -(chosen.log_prob(seen["actions"].long()) * advantage).mean()
    return actor + 0.5 * (returns - values).square().mean() - 0.01 * chosen.entropy().mean(), logits


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--envs", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--updates", type=int, default=10)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    args = ap.parse_args()
    torch.manual_seed(0)
    sim = cx.Craftax(args.envs, cx.default_config(obs_mode=cx.OBS_SYM_F32))
    sim.reset(synth.seeds_for(args.envs))
    policy = Policy(sim.obs_bytes // 4, dtype={"bf16": torch.bfloat16, "f32": torch.float32}[args.dtype])
    optimizer = torch.optim.Adam(policy.parameters(), lr=3e-4, eps=1e-5)
    states, first = policy.empty(args.envs), torch.ones(args.envs, dtype=torch.uint8, device="cuda")
    for update in range(args.updates):
        began = [[v.clone() for v in state] for state in states]
        seen = act(policy, sim, states, first, args.steps)
        loss, logits = loss_of(policy, seen, began)
        optimizer.zero_grad(set_to_none=True)
        loss.backward()
        torch.nn.utils.clip_grad_norm_(policy.parameters(), 0.5)
        optimizer.step()
        print(f"update {update}: reward a step {float(seen['reward'].mean()):.5f}, loss {float(loss.detach()):.4f}, "
              f"logits of the two forms {float((logits.detach() - seen['logits']).abs().max()):.2g} apart", flush=True)
    sim.close()


if __name__ == "__main__":
    main()

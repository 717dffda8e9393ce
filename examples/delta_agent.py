"""A search agent whose memory is a matrix, and a smaller one that learns from it: python examples/delta_agent.py

The agent of search_agent.py (Sec. 4.1 of the paper: three directions per knob, clipped policy gradient, value head, entropy bonus) with another shared
layer: the gated delta rule over the steps of an episode, whose state holds what followed which configuration.

  rollout    gated_delta of one step keeps the layer's state in place, sample draws an action per knob, apply_actions moves the configurations,
             gbt_score predicts their fitness
  training   gated_delta over whole episodes, token_logprobs for the log-probabilities of the actions taken and the entropy, AdamW
  teaching   token_logprobs lists the agent's best directions, distill_loss brings a smaller agent's distribution to them
"""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_1905_12799_amd import binding as rls        # noqa: E402
from paper_1905_12799_amd import synth                 # noqa: E402

GAMMA, LAMBDA, CLIP, VALUE, ENTROPY, EPOCHS, LR, MAX_NORM = 0.9, 0.99, 0.3, 1.0, 0.1, 3, 1e-3, 0.5
DIRECTIONS, LISTED = 3, 2


class DeltaAgent:
    """heads of value_dim values each; two heads share a key head."""

    def __init__(self, knobs, heads, key_dim, value_dim, generator):
        def init(*shape):
            return (torch.randn(*shape, generator=generator) / shape[-1] ** 0.5).cuda().requires_grad_()
        self.knobs, self.heads, self.key_dim, self.value_dim = knobs, heads, key_dim, value_dim
        self.key_heads = max(1, heads // 2)
        inputs, width = knobs + 1, heads * value_dim
        self.params = [init(self.key_heads * key_dim, inputs), init(self.key_heads * key_dim, inputs), init(width, inputs), init(2 * heads, inputs),
                       init(DIRECTIONS * knobs, width), init(1, width)]
        self.optimizer = rls.AdamW([p.detach() for p in self.params])

    def empty_state(self, n):
        return torch.zeros(n, self.heads, self.key_dim, self.value_dim, device="cuda")

    def inputs(self, x):
        """What the layer takes of configurations [..., knobs]: q, k of length 1, v, logarithms of the decay, beta."""
        x = torch.cat([x, torch.ones_like(x[..., :1])], -1)
        wq, wk, wv, wg = self.params[:4]
        unit = torch.nn.functional.normalize
        q, k = (unit((x @ w.t()).unflatten(-1, (self.key_heads, self.key_dim)), dim=-1) for w in (wq, wk))
        gates = x @ wg.t()
        return q, k, (x @ wv.t()).unflatten(-1, (self.heads, self.value_dim)), -torch.nn.functional.softplus(gates[..., :self.heads] - 2).contiguous(), \
            torch.sigmoid(gates[..., self.heads:]).contiguous()

    def heads_of(self, o):
        wp, wv = self.params[4:]
        o = o.flatten(-2)
        return (o @ wp.t()).unflatten(-1, (self.knobs, DIRECTIONS)), (o @ wv.t())[..., 0]

    def forward(self, x, layer=rls.gated_delta):
        """Logits [n, steps, knobs, 3] and values of whole episodes [n, steps, knobs]."""
        return self.heads_of(layer(*self.inputs(x))[0])

    def step(self, loss):
        grads = [torch.zeros_like(p) if g is None else g.contiguous() for p, g in zip(self.params, torch.autograd.grad(loss, self.params, allow_unused=True))]
        norm = torch.stack([g.square().sum() for g in grads]).sum().sqrt()
        self.optimizer.step(grads, lr=LR, weight_decay=0.0, grad_scale=(MAX_NORM / (norm + 1e-6)).clamp(max=1.0).reshape(1))


@torch.no_grad()
def rollout(agent, cfg, sizes, domains, forest, steps, generator):
    n, knobs = cfg.shape
    state = agent.empty_state(n)
    xs, actions, logps, values, scores = [], [], [], [], []
    first = rls.gbt_score(forest, cfg.float()).clone()
    for _ in range(steps):
        x = cfg.float() / sizes * 2 - 1
        o, _ = rls.gated_delta(*agent.inputs(x[:, None]), state=state, last=state)         # one step, the state in place
        logits, value = agent.heads_of(o[:, 0])
        token, logp = rls.sample(logits.reshape(n * knobs, DIRECTIONS), torch.rand(n * knobs, device="cuda", generator=generator))
        cfg, feats = rls.apply_actions(cfg, (token - 1).to(torch.int8).view(n, knobs), domains)
        xs.append(x), actions.append(token.view(n, knobs)), logps.append(logp.view(n, knobs).sum(1)), values.append(value)
        scores.append(rls.gbt_score(forest, feats).clone())
    scores = torch.stack(scores, 1)
    rewards = scores - torch.cat([first[:, None], scores[:, :-1]], 1)
    return (torch.stack(xs, 1), torch.stack(actions, 1), torch.stack(logps, 1), torch.stack(values, 1), rewards), scores


def policy_loss(agent, batch, advantage, returns, layer=rls.gated_delta, logprobs=rls.token_logprobs):
    xs, actions, logps, _, _ = batch
    logits, value = agent.forward(xs, layer)
    r = logprobs(logits.reshape(-1, DIRECTIONS), actions.reshape(-1).contiguous())
    ratio = torch.exp(r.logprob.view(actions.shape).sum(-1) - logps)
    gain = torch.minimum(ratio * advantage, ratio.clamp(1 - CLIP, 1 + CLIP) * advantage).mean()
    return -gain + VALUE * (value - returns).square().mean() - ENTROPY * r.entropy.mean()


def advantages(batch):
    _, _, _, values, rewards = batch
    following = torch.cat([values[:, 1:], torch.zeros_like(values[:, :1])], 1)
    discount = torch.full((1, 1, 1), GAMMA * LAMBDA, device="cuda").expand(*values.shape, 1)
    advantage = rls.linear_scan(discount, (rewards + GAMMA * following - values)[:, :, None], reverse=True)[0][:, :, 0]
    return (advantage - advantage.mean()) / (advantage.std() + 1e-6), advantage + values


def train(agent, batch):
    advantage, returns = advantages(batch)
    for _ in range(EPOCHS):
        agent.step(policy_loss(agent, batch, advantage, returns))


def taught_by(teacher, xs):
    """The teacher's best directions, of every knob and step, and their log-probabilities."""
    with torch.no_grad():
        r = rls.token_logprobs(teacher.forward(xs)[0].reshape(-1, DIRECTIONS), None, top=LISTED)
    return r.top_token, r.top_logprob


def teaching_loss(student, xs, tokens, logprobs, layer=rls.gated_delta, distill=rls.distill_loss):
    return distill(student.forward(xs, layer)[0].reshape(-1, DIRECTIONS), tokens, logprobs)[0].mean()


def main(rounds=20, configurations=1024, steps=64, heads=4, key_dim=32, value_dim=32, seed=12799, verbose=True):
    """Trains the agent and teaches a smaller one; returns the mean predicted fitness at the end of each round's episodes, and the losses of the teaching."""
    generator = torch.Generator().manual_seed(seed)
    draws = torch.Generator(device="cuda").manual_seed(seed)
    space = synth.conv2d_knob_space(128, 128, 28, 3)
    domains = rls.DeviceDomains(*space.domains_csr())
    sizes = torch.tensor(space.sizes, dtype=torch.float32).cuda()
    problem = synth.make_problem(synth.WORKLOADS["tiny"])
    knobs = len(space.sizes)
    forest_rows = (torch.rand(4096, knobs, generator=generator) * sizes.cpu()).floor().numpy()
    forest = rls.DeviceForest.from_host(synth.random_forest(forest_rows, problem.forest.n_trees, problem.forest.depth, knobs, np.random.default_rng(seed)))
    agent = DeltaAgent(knobs, heads, key_dim, value_dim, generator)
    student = DeltaAgent(knobs, max(1, heads // 2), key_dim // 2, value_dim // 2, generator)
    fitness, losses = [], []
    for k in range(rounds):
        start = (torch.rand(configurations, knobs, device="cuda", generator=draws) * sizes).floor().to(torch.int32)
        batch, scores = rollout(agent, start, sizes, domains, forest, steps, draws)
        train(agent, batch)
        for _ in range(EPOCHS):
            loss = teaching_loss(student, batch[0], *taught_by(agent, batch[0]))
            student.step(loss)
        fitness.append(float(scores[:, -1].mean()))
        losses.append(float(loss.detach()))
        if verbose:
            print(f"round {k}: mean predicted fitness {fitness[-1]:.3f}, best {float(scores.max()):.3f}; the student's divergence {losses[-1]:.4f}", flush=True)
    return fitness, losses


if __name__ == "__main__":
    main()

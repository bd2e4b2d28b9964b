"""A policy with a mixture-of-experts block, trained for a few steps on one GPU.

    python examples/expert_policy.py [--steps 20]

Per step: layer norm, a router (torch), the experts' two products around a
squared ReLU, layer norm, logits, the clipped policy loss with its KL term,
the backward pass, and one step of TurboMuon on the experts' matrices and the
head (the vectors, the embedding and the router go to SGD).  The task is a toy
one: the advantage of a sampled token is 1 where it is the successor of the
token before it, -1 otherwise, so the share of right tokens has to rise.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2512_04632_amd import ops  # noqa: E402
from paper_2512_04632_amd.optim import TurboMuon  # noqa: E402


class ExpertPolicy(torch.nn.Module):
    def __init__(self, vocab=512, dim=256, hidden=512, experts=8):
        super().__init__()

        def param(*shape, scale):
            return torch.nn.Parameter(torch.randn(shape) * scale)

        self.embed = param(vocab, dim, scale=1.0)
        self.norm_in = torch.nn.ParameterList([torch.ones(dim), torch.zeros(dim)])
        self.norm_out = torch.nn.ParameterList([torch.ones(dim), torch.zeros(dim)])
        self.router = param(dim, experts, scale=dim ** -0.5)
        self.up = param(experts, dim, hidden, scale=dim ** -0.5)
        self.down = param(experts, hidden, dim, scale=hidden ** -0.5)
        self.head = param(1, dim, vocab, scale=dim ** -0.5)

    def matrices(self):
        return [self.up, self.down, self.head]

    def vectors(self):
        return [self.embed, self.router, *self.norm_in, *self.norm_out]

    def forward(self, tokens):
        x = self.embed[tokens].bfloat16()
        h = ops.layer_norm(x, *self.norm_in)
        share, expert = (h.float() @ self.router).softmax(-1).max(-1)
        order = expert.argsort(stable=True)
        ends = torch.bincount(expert, minlength=self.up.shape[0]).cumsum(0).to(torch.int32)
        a = ops.expert_linear(h[order], self.up, ends)
        y = ops.expert_linear(a.relu().square(), self.down, ends)
        back = torch.empty_like(order).scatter_(0, order, torch.arange(len(order), device=order.device))
        x = x + y[back] * share[:, None].bfloat16()
        h = ops.layer_norm(x, *self.norm_out)
        everyone = torch.full((1,), len(tokens), dtype=torch.int32, device=tokens.device)
        return ops.expert_linear(h, self.head, everyone)   # one matrix for every row


def train(steps=20, rows=4096, vocab=512, seed=0, say=print):
    """Runs the steps; returns the share of right tokens among the samples of each."""
    torch.manual_seed(seed)
    policy = ExpertPolicy(vocab=vocab).cuda()
    muon = TurboMuon(policy.matrices(), lr=0.02)
    sgd = torch.optim.SGD(policy.vectors(), lr=0.1)
    right = []
    for step in range(steps):
        tokens = torch.randint(vocab, (rows,), device="cuda")
        with torch.no_grad():
            logits = policy(tokens).float()
            # half of the samples are the wanted token, as from a replayed good answer
            sampled = torch.multinomial(logits.softmax(-1), 1)[:, 0]
            wanted = (tokens + 1) % vocab
            taken = torch.where(torch.rand(rows, device="cuda") < 0.5, wanted, sampled)
            old = logits.log_softmax(-1).gather(-1, taken[:, None])[:, 0]
        advantage = torch.where(taken == wanted, 1.0, -1.0)
        weights = torch.full((rows,), 1.0 / rows, device="cuda")
        right.append(float((sampled == wanted).float().mean()))
        for _ in range(2):   # two updates on the same samples, so that ratios leave one
            muon.zero_grad()
            sgd.zero_grad()
            loss, _ = ops.policy_loss(policy(tokens), taken, old, advantage, weights, ref_logp=old, kl=0.01)
            loss.backward()
            muon.step()
            sgd.step()
        say(f"step {step:3d}  loss {float(loss.detach()):+.4f}  right {right[-1]:.3f}")
    return right


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    parser.add_argument("--steps", type=int, default=20)
    train(parser.parse_args().steps)

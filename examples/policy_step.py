"""Trains a one-layer mixture-of-experts policy on rewards: answering a few requests, scoring what was answered and a clipped step of all
gradients, as a loop of reinforcement learning uses them.

    python examples/policy_step.py [steps]

Answering: the experts on a few tokens (``experts.layer``), the likeliest next tokens with their log probabilities (``LossHead.log_probs``),
one of them drawn.  Learning: the tokens to their experts and back (``experts``), log probabilities and entropies of the answers with their
gradients (``log_probs``, ``log_probs_backward``), the norm of all gradients (``clipping.GradClipper``) and the steps that take its scale
(``MuonStepper``, ``muon_adamw_step``).  torch supplies memory, the experts' own products in training and elementwise glue.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2502_16982_amd import binding, clipping, experts, losses  # noqa: E402

VOCAB, WIDTH, INNER, EXPERTS, TOP = 1009, 128, 96, 8, 2
REQUESTS, ROUNDS, ALTERNATIVES = 32, 16, 16
ENTROPY, MAX_NORM = 0.01, 0.5


class Policy:
    def __init__(self, device, seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, std):
            return (torch.randn(*shape, generator=gen, device=device) * std).to(torch.bfloat16)

        self.embed, self.head, self.router = normal(VOCAB, WIDTH, std=1.0), normal(VOCAB, WIDTH, std=0.02), normal(WIDTH, EXPERTS, std=0.09)
        self.up, self.gate = normal(EXPERTS, WIDTH, INNER, std=0.09), normal(EXPERTS, WIDTH, INNER, std=0.09)
        self.down = normal(EXPERTS, INNER, WIDTH, std=0.1)
        self.params = {"embed": self.embed, "head": self.head, "router": self.router, "up": self.up, "gate": self.gate, "down": self.down}
        self.grads = {name: torch.zeros_like(p) for name, p in self.params.items()}
        matrices = [(self.router, self.grads["router"])]
        for name in ("up", "gate", "down"):                # each expert's matrix is one of its own to the optimizer
            matrices += zip(self.params[name], self.grads[name])
        self.stepper = binding.MuonStepper([(w, g, torch.zeros_like(w, dtype=torch.float32)) for w, g in matrices])
        self.adam = [(self.params[n], self.grads[n], *(torch.zeros_like(self.params[n], dtype=torch.float32) for _ in range(2)))
                     for n in ("embed", "head")]
        self.clipper = clipping.GradClipper(self.grads.values())
        self.answers = losses.LossHead(REQUESTS, VOCAB, WIDTH, gradients=False)
        self.scores = losses.LossHead(REQUESTS * ROUNDS, VOCAB, WIDTH)
        self.steps = 0

    def route(self, x):
        score, chosen = (x @ self.router).float().topk(TOP, dim=1)
        return chosen, score.softmax(1)

    def answer(self, tokens, gen=None):
        """A next token for each of a few, drawn from the likeliest."""
        x = self.embed[tokens]
        chosen, weights = self.route(x)
        hidden = x + experts.layer(x, self.up, self.down, chosen, weights, gate=self.gate)
        s = self.answers.log_probs(hidden, self.head, top=ALTERNATIVES)
        pick = torch.multinomial(s.top_log_prob.exp(), 1, generator=gen)
        return s.top_index.gather(1, pick)[:, 0]

    def learn(self, tokens, answers, d_log_prob, d_entropy):
        """Gradients of sum(d_log_prob * log_prob + d_entropy * entropy) into ``grads``; the scores."""
        x = self.embed[tokens]
        chosen, weights = self.route(x)
        routing = experts.sort_by_expert(chosen, EXPERTS)
        rows = experts.dispatch(x, routing)
        edges = routing.offsets.tolist()
        lead, inner, y = rows.new_empty(rows.shape[0], INNER), rows.new_empty(rows.shape[0], INNER), torch.empty_like(rows)
        for e, (a, b) in enumerate(zip(edges, edges[1:])):
            torch.mm(rows[a:b], self.gate[e], out=lead[a:b])
            torch.mm(rows[a:b], self.up[e], out=inner[a:b])
        share = lead.float().sigmoid()
        act = lead * share
        h = (act * inner).to(rows.dtype)
        for e, (a, b) in enumerate(zip(edges, edges[1:])):
            torch.mm(h[a:b], self.down[e], out=y[a:b])
        hidden = x + experts.combine(y, weights, routing)

        s = self.scores.log_probs(hidden, self.head, answers)
        d_hidden, d_head = self.scores.log_probs_backward(hidden, self.head, answers, s, d_log_prob, d_entropy)
        self.grads["head"].copy_(d_head)

        d_y, d_weights = experts.combine_backward(d_hidden, y, weights, routing)
        d_rows, d_h = torch.empty_like(rows), torch.empty_like(h)
        for e, (a, b) in enumerate(zip(edges, edges[1:])):
            torch.mm(h[a:b].T, d_y[a:b], out=self.grads["down"][e])
            torch.mm(d_y[a:b], self.down[e].T, out=d_h[a:b])
        d_inner = (d_h * act).to(rows.dtype)
        d_lead = (d_h * inner * share * (1 + lead * (1 - share))).to(rows.dtype)
        for e, (a, b) in enumerate(zip(edges, edges[1:])):
            torch.mm(rows[a:b].T, d_inner[a:b], out=self.grads["up"][e])
            torch.mm(rows[a:b].T, d_lead[a:b], out=self.grads["gate"][e])
            torch.addmm(d_inner[a:b] @ self.up[e].T, d_lead[a:b], self.gate[e].T, out=d_rows[a:b])
        d_score = weights * (d_weights - (weights * d_weights).sum(1, keepdim=True))
        d_score = torch.zeros(tokens.numel(), EXPERTS, device=x.device).scatter_(1, chosen, d_score).to(x.dtype)
        torch.mm(x.T, d_score, out=self.grads["router"])
        d_x = d_hidden + experts.dispatch_backward(d_rows, routing) + d_score @ self.router.T
        self.grads["embed"].zero_().index_add_(0, tokens, d_x)
        return s

    def step(self, tokens, answers, reward):
        """One step on answers and their rewards; the gradients' norm before it was clipped, the mean entropy."""
        n = tokens.numel()
        advantage = reward - reward.mean()
        s = self.learn(tokens, answers, -advantage / n, torch.full((n,), -ENTROPY / n, device=tokens.device))
        clip = self.clipper.scale(MAX_NORM)
        self.steps += 1
        self.stepper.step(binding.default_hparams(lr=0.005, weight_decay=0.0), grad_scale=clip.scale)
        binding.muon_adamw_step(self.adam, lr=0.005, weight_decay=0.0, step=self.steps, grad_scale=clip.scale,
                                stream_ptr=torch.cuda.current_stream(tokens.device).cuda_stream)
        return clip.norm, s.entropy.mean()


def wanted(tokens, answers):
    """Reward: answers from the half of the vocabulary that the request's number names."""
    return ((tokens + answers) % 2 == 0).float()


def train(steps, device="cuda:0", report=None):
    policy, gen = Policy(device), torch.Generator(device=device).manual_seed(1)
    history = []
    for i in range(steps):
        tokens = torch.randint(VOCAB, (ROUNDS, REQUESTS), generator=gen, device=device)
        answers = torch.stack([policy.answer(t, gen) for t in tokens])
        reward = wanted(tokens, answers)
        norm, entropy = policy.step(tokens.reshape(-1), answers.reshape(-1), reward.reshape(-1))
        if i % 10 == 0 or i == steps - 1:
            history.append((i, float(reward.mean()), float(entropy), float(norm)))
            if report:
                report(*history[-1])
    return history


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 100,
          report=lambda i, reward, entropy, norm: print(f"step {i:4d}  reward {reward:.3f}  entropy {entropy:.3f}  gradient norm {norm:.4f}", flush=True))

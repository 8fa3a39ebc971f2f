"""Trains a one-layer mixture-of-experts language model on synthetic text: the head's losses, the experts' dispatch and the
optimizer step together, as a training loop uses them.

    python examples/mixture_step.py [steps]

Forward: embedding, router, tokens to their experts and back (``experts``), head.  Losses: cross entropy against the next token and
distillation from a teacher's four best logits (``losses``).  The gradients go to ``MuonStepper`` (experts' matrices and router) and to
``muon_adamw_step`` (embedding and head, which stay off Muon).  torch supplies memory, the experts' own products and elementwise glue.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2502_16982_amd import binding, experts, losses  # noqa: E402

VOCAB, WIDTH, INNER, EXPERTS, TOP, TOKENS = 4001, 256, 128, 16, 2, 1024
SHARE = 0.5                       # of the distillation in the training loss


class Mixture:
    def __init__(self, device, seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, std=0.02):
            return (torch.randn(*shape, generator=gen, device=device) * std).to(torch.bfloat16)

        self.embed, self.head = normal(VOCAB, WIDTH, std=1.0), normal(VOCAB, WIDTH)
        self.router = normal(WIDTH, EXPERTS, std=0.06)
        self.up = [normal(WIDTH, INNER, std=0.06) for _ in range(EXPERTS)]
        self.down = [normal(INNER, WIDTH, std=0.09) for _ in range(EXPERTS)]
        matrices = [self.router, *self.up, *self.down]
        self.grads = [torch.zeros_like(w) for w in matrices]
        self.stepper = binding.MuonStepper([(w, g, torch.zeros_like(w, dtype=torch.float32)) for w, g in zip(matrices, self.grads)])
        self.adam = [(p, torch.zeros_like(p), torch.zeros_like(p, dtype=torch.float32), torch.zeros_like(p, dtype=torch.float32))
                     for p in (self.embed, self.head)]
        self.loss_head = losses.LossHead(TOKENS, VOCAB, WIDTH)
        self.steps = 0

    def step(self, tokens, targets, teacher_index, teacher_logits):
        """One training step; the two mean losses."""
        # forward
        x = self.embed[tokens]
        score, chosen = (x @ self.router).float().topk(TOP, dim=1)
        weights = score.softmax(1)
        routing = experts.sort_by_expert(chosen, EXPERTS)
        rows = experts.dispatch(x, routing)
        edges = routing.offsets.tolist()
        inner, y = rows.new_empty(rows.shape[0], INNER), torch.empty_like(rows)
        for e, (a, b) in enumerate(zip(edges, edges[1:])):
            torch.mm(rows[a:b], self.up[e], out=inner[a:b])
            torch.mm(inner[a:b].relu(), self.down[e], out=y[a:b])
        hidden = x + experts.combine(y, weights, routing)

        # losses and the gradients of the head's inputs
        scale = torch.full((tokens.numel(),), (1 - SHARE) / tokens.numel(), device=x.device)
        ce = self.loss_head.cross_entropy(hidden, self.head, targets, token_scale=scale)
        kd = self.loss_head.distill(hidden, self.head, teacher_index, teacher_logits, temperature=2.0,
                                    token_scale=scale * (SHARE / (1 - SHARE)))
        d_hidden = ce.d_hidden + kd.d_hidden
        torch.add(ce.d_weight, kd.d_weight, out=self.adam[1][1])

        # backward through the mixture
        d_y, d_weights = experts.combine_backward(d_hidden, y, weights, routing)
        d_rows = torch.empty_like(rows)
        for e, (a, b) in enumerate(zip(edges, edges[1:])):
            torch.mm(inner[a:b].relu().T, d_y[a:b], out=self.grads[1 + EXPERTS + e])
            d_inner = (d_y[a:b] @ self.down[e].T) * (inner[a:b] > 0)
            torch.mm(rows[a:b].T, d_inner, out=self.grads[1 + e])
            torch.mm(d_inner, self.up[e].T, out=d_rows[a:b])
        d_score = weights * (d_weights - (weights * d_weights).sum(1, keepdim=True))
        d_score = torch.zeros(tokens.numel(), EXPERTS, device=x.device).scatter_(1, chosen, d_score).to(x.dtype)
        torch.mm(x.T, d_score, out=self.grads[0])
        d_x = d_hidden + experts.dispatch_backward(d_rows, routing) + d_score @ self.router.T
        self.adam[0][1].zero_().index_add_(0, tokens, d_x)

        # the optimizer's step
        self.steps += 1
        self.stepper.step(binding.default_hparams(lr=0.01, weight_decay=0.0))
        binding.muon_adamw_step(self.adam, lr=0.01, weight_decay=0.0, step=self.steps,
                                stream_ptr=torch.cuda.current_stream(x.device).cuda_stream)
        return ce.loss.mean(), kd.loss.mean()


def batch(device, gen):
    """Text in which a token is followed by one of four, the first of them half of the time, and a teacher that knows."""
    tokens = torch.randint(VOCAB, (TOKENS,), generator=gen, device=device)
    follow = (tokens[:, None] * 31 + torch.tensor([7, 1009, 2003, 3001], device=device)) % VOCAB
    share = torch.tensor([0.5, 0.25, 0.15, 0.1], device=device)
    pick = torch.multinomial(share.expand(TOKENS, 4), 1, generator=gen)
    return tokens, follow.gather(1, pick)[:, 0], follow, share.log().expand(TOKENS, 4).contiguous()


def train(steps, device="cuda:0", report=None):
    model, gen = Mixture(device), torch.Generator(device=device).manual_seed(1)
    history = []
    for i in range(steps):
        ce, kd = model.step(*batch(device, gen))
        if i % 10 == 0 or i == steps - 1:
            history.append((i, float(ce), float(kd)))
            if report:
                report(*history[-1])
    return history


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 100,
          report=lambda i, ce, kd: print(f"step {i:4d}  cross entropy {ce:.3f}  distillation {kd:.3f}", flush=True))

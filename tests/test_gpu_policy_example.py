"""The policy example: it runs, its gradients are those of torch's autograd in fp64 on the same parameters, and what it answers with and what it learns
with are one network.

bf16 rounds every stored intermediate (2^-8 at most, about 2^-9.5 as a root mean square); some ten of them in a row, independent, stay below 2e-2 of a
gradient as a whole.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    from examples import policy_step
    return policy_step


def reference(policy, params, tokens, chosen):
    """(log probabilities of the whole vocabulary) in fp64 with given experts."""
    x = params["embed"][tokens]
    weights = (x @ params["router"]).gather(1, chosen).softmax(1)
    hidden = x
    for j in range(chosen.shape[1]):
        pick = chosen[:, j]
        lead = torch.bmm(x[:, None], params["gate"][pick])[:, 0]
        inner = lead * torch.sigmoid(lead) * torch.bmm(x[:, None], params["up"][pick])[:, 0]
        hidden = hidden + weights[:, j:j + 1] * torch.bmm(inner[:, None], params["down"][pick])[:, 0]
    return torch.log_softmax(hidden @ params["head"].T, 1)


def test_gradients(example):
    policy = example.Policy("cuda:0", seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    n = 300
    tokens = torch.randint(example.VOCAB, (n,), generator=gen, device="cuda")
    answers = torch.randint(example.VOCAB, (n,), generator=gen, device="cuda")
    dl, de = torch.randn(n, generator=gen, device="cuda") / n, torch.full((n,), 0.2 / n, device="cuda")
    s = policy.learn(tokens, answers, dl, de)
    chosen, _ = policy.route(policy.embed[tokens])
    params = {name: p.double().cpu().requires_grad_() for name, p in policy.params.items()}
    logp = reference(policy, params, tokens.cpu(), chosen.cpu())
    given, entropy = logp.gather(1, answers.cpu()[:, None])[:, 0], -(logp.exp() * logp).sum(1)
    (dl.double().cpu() * given + de.double().cpu() * entropy).sum().backward()
    assert (s.log_prob.double().cpu() - given).norm() <= 1e-2 * given.norm()
    for name, p in params.items():
        got = policy.grads[name].double().cpu()
        assert (got - p.grad).norm() <= 2e-2 * p.grad.norm(), name
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in policy.grads.values()))
    assert abs(float(policy.clipper.scale(1.0).norm) - norm) <= 1e-12 * norm


def test_answers_come_from_the_network_that_learns(example):
    """The few tokens' way and the sorted one give the same distribution."""
    policy = example.Policy("cuda:0", seed=5)
    tokens = torch.arange(example.REQUESTS, device="cuda")
    answers = policy.answer(tokens, torch.Generator(device="cuda").manual_seed(6))
    zero = torch.zeros(example.REQUESTS, device="cuda")
    s = policy.learn(tokens, answers, zero, zero)
    chosen, weights = policy.route(policy.embed[tokens])
    from paper_2502_16982_amd import experts
    hidden = policy.embed[tokens] + experts.layer(policy.embed[tokens], policy.up, policy.down, chosen, weights, gate=policy.gate)
    few = policy.answers.log_probs(hidden, policy.head, answers, top=example.ALTERNATIVES)
    assert (few.log_prob - s.log_prob).abs().max() <= 2e-2 and (few.entropy - s.entropy).abs().max() <= 2e-2
    assert (few.top_index == answers[:, None]).any(1).all()
    assert all((g == 0).all() for g in policy.grads.values())


def test_runs(example):
    history = example.train(3)
    assert len(history) == 2 and all(math.isfinite(v) for row in history for v in row)

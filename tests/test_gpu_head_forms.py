"""Forms of the head's calls that leave something out, against the call that has it: forward only, one gradient, no log of the sum."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as ho

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def losses():
    from paper_2502_16982_amd import losses as l
    return l


def make(tokens, vocab, width, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(vocab, width, generator=g) * 0.05
    h = torch.randn(tokens, width, generator=g)
    return h.to(DT[dtype]).cuda(), w.to(DT[dtype]).cuda(), g


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("top", [1, 2, 3, 4, 5, 9, 70])
@pytest.mark.parametrize("tokens,vocab,width", [(1, 7, 8), (19, 300, 72), (130, 1027, 100), (17, 9000, 200)])
def test_distillation_without_gradients(losses, dtype, top, tokens, vocab, width):
    """Up to four entries the join makes their logits itself.  Loss and lse within the errors of two sums of `width` products, (4 + sqrt(D))
    2^-23 A each, A the largest sum of |h w| of the token over tau, and roundings of their own size."""
    h, w, g = make(tokens, vocab, width, dtype, seed=top)
    index, s = torch.randint(vocab, (tokens, top), generator=g), torch.randn(tokens, top, generator=g) * 2
    none = torch.rand(tokens, top, generator=g)
    index[none < 0.15] = -1
    s[(none >= 0.15) & (none < 0.3)] = -float("inf")
    index[:1], s[:1] = torch.arange(top) % vocab, torch.arange(top) * 0.1
    if tokens > 3:
        index[2], index[3, -1] = -1, vocab                  # no entry; an index beyond the vocabulary
    tau = 1.5
    head = losses.LossHead(tokens, vocab, width, DT[dtype])
    r = head.distill(h, w, index.cuda(), s.cuda(), temperature=tau, gradients=False)
    assert r.d_hidden is None and r.d_weight is None
    h64, w64 = (t.double().cpu().numpy() for t in (h, w))
    want = ho.head_loss(h64, w64, index=index.numpy(), teacher=s.double().numpy(), tau=tau)
    off = (4 + np.sqrt(width)) * 2.0 ** -23 * (np.abs(h64) @ np.abs(w64).T).max(axis=1) / tau + 2.0 ** -21 + 2.0 ** -22 * np.abs(want["lse"])
    loss, lse = r.loss.double().cpu().numpy(), r.lse.double().cpu().numpy()
    assert (np.abs(lse - want["lse"]) <= off).all()
    assert np.array_equal(np.isnan(loss), np.isnan(want["loss"]))
    ok = ~np.isnan(loss)
    assert (np.abs(loss - want["loss"])[ok] <= (tau * tau * (2 * off + 2.0 ** -22 * 10 / tau) + 2.0 ** -23 * np.abs(want["loss"]))[ok]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", [(3, 129, 24), (300, 2050, 520), (64, 9001, 256)])
def test_one_gradient_alone(losses, dtype, tokens, vocab, width):
    h, w, g = make(tokens, vocab, width, dtype)
    index, s = torch.randint(vocab, (tokens, 6), generator=g).cuda(), torch.randn(tokens, 6, generator=g).cuda()
    scale = torch.rand(tokens, generator=g).cuda()
    head = losses.LossHead(tokens, vocab, width, DT[dtype])
    for call in (lambda k: head.cross_entropy(h, w, index[:, 0].contiguous(), token_scale=scale, gradients=k),
                 lambda k: head.distill(h, w, index, s, temperature=2.0, token_scale=scale, gradients=k)):
        both, hidden, weight = call(True), call(("hidden",)), call(["weight"])
        assert hidden.d_weight is None and torch.equal(hidden.d_hidden, both.d_hidden)
        assert weight.d_hidden is None and torch.equal(weight.d_weight, both.d_weight)
        assert torch.equal(hidden.loss, both.loss) and torch.equal(weight.loss, both.loss)

"""Values at the edge of what the head's losses take, each against the same call written without them."""
import pytest
import torch

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


@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("teacher", ["bf16", "f32"])
@pytest.mark.parametrize("top", [3, 70])
def test_lowest_teacher_logits(losses, tau, teacher, top):
    """A logit of the type's lowest value is a finite one: beside others it has no weight, but a token whose entries all hold it has them
    all alike, whatever the temperature.  Tokens with equal weights on equal entries agree bit for bit.  An entry without weight takes its
    probability from a dot product and what is no entry from the matrix product: each is off by (4 + sqrt(D)) 2^-23 A + 2^-21
    relative (A: largest sum of |h w| over tau), which the gradients carry times tau |w| and |h|."""
    h, w, g = make(6, 200, 64, "f32")
    index = torch.stack([torch.randperm(200, generator=g)[:top] for _ in range(6)]).cuda()
    s = torch.randn(6, top, generator=g).to(DT[teacher]).cuda()
    same, low = s.clone(), torch.finfo(DT[teacher]).min
    s[1], same[1] = low, 0.0                                 # all alike
    s[2, ::2], same[2, ::2] = low, -float("inf")             # masked
    s[3], same[3] = -low, 0.0                                # the highest value, all alike
    s[4, 1:], same[4, 1:] = low, -float("inf")
    head = losses.LossHead(6, 200, 64, torch.float32)
    a, b = (head.distill(h, w, index, x, temperature=tau) for x in (s, same))
    assert (a.loss[1] != 0) and torch.isfinite(a.loss).all()
    assert torch.equal(a.loss, b.loss) and torch.equal(a.lse, b.lse)
    alike = [0, 1, 3, 5]
    assert torch.equal(a.d_hidden[alike], b.d_hidden[alike])
    off = 2 * tau * (12 * 2.0 ** -23 * float(h.abs().mm(w.abs().T).max()) / tau + 2.0 ** -21)
    assert (a.d_hidden - b.d_hidden).abs().max() <= off * w.abs().max()
    assert (a.d_weight - b.d_weight).abs().max() <= off * h.abs().sum(0).max()

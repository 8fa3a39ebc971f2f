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


def want64(h, w, y, scale):
    """loss, d_hidden and d_weight of cross entropy in fp64 on the device; tokens with y < 0 or y >= vocab have no gradient."""
    h64, w64, there = h.double(), w.double(), (y >= 0) & (y < len(w))
    z = torch.mm(h64, w64.T.contiguous())
    lse = torch.logsumexp(z, 1)
    at = torch.where(there, y, 0)[:, None]
    dz = (z - lse[:, None]).exp()
    dz.scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None])
    dz *= torch.where(there, scale.double(), 0.0)[:, None]
    return torch.where(there, lse - z.gather(1, at)[:, 0], 0.0), torch.mm(dz, w64), torch.mm(dz.T.contiguous(), h64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("limit", [0, 1, 8 << 30])
@pytest.mark.parametrize("tokens", [70, 700, 20000])
def test_scales_of_tokens_without_gradient_do_not_matter(losses, dtype, limit, tokens):
    """Tokens with scales of their own, in one piece (with more than 16384 tokens the largest scale is found in a launch of its own) and in
    many.  Ignored ones and those with a target beyond the vocabulary may have any scale: the others' gradients do not notice.  Against
    fp64: bf16 rounds dz and the result once each, 5e-3 of a row or of the whole; fp32 1e-5."""
    h, w, g = make(tokens, 50, 24, dtype)
    y = torch.randint(50, (tokens,), generator=g).cuda()
    scale = (torch.rand(tokens, generator=g) * 3 + 0.01).cuda() / tokens
    y[3::7], y[5::11] = -100, 50
    head = losses.LossHead(tokens, 50, 24, DT[dtype], max_workspace_bytes=limit)
    gone = (y < 0) | (y >= 50)
    a = head.cross_entropy(h, w, y, token_scale=torch.where(gone, 0.0, scale))
    b = head.cross_entropy(h, w, y, token_scale=torch.where(gone, torch.finfo(torch.float32).max, scale))
    assert torch.equal(torch.isnan(a.loss), y >= 50) and torch.equal(a.loss.nan_to_num(), b.loss.nan_to_num())
    assert torch.equal(a.d_hidden, b.d_hidden) and torch.equal(a.d_weight, b.d_weight)
    loss, d_hidden, d_weight = want64(h, w, y, scale)
    bar = 5e-3 if dtype == "bf16" else 1e-5
    assert (a.loss.nan_to_num() - loss).abs().max() <= 1e-5
    assert not a.d_hidden[gone].any()
    # a row of 24 elements has fewer roundings to average: twice the bar
    assert ((a.d_hidden - d_hidden).norm(dim=1) <= 2 * bar * d_hidden.norm(dim=1)).all()
    assert (a.d_weight - d_weight).norm() <= bar * d_weight.norm()


@pytest.mark.parametrize("limit", [0, 1])
def test_scales_of_a_distillation(losses, limit):
    h, w, g = make(700, 50, 24, "f32")
    index, s = torch.randint(50, (700, 3), generator=g).cuda(), torch.randn(700, 3, generator=g).cuda()
    index[::5], s[1::5] = -1, -float("inf")
    scale = torch.rand(700, generator=g).cuda() + 0.1
    head = losses.LossHead(700, 50, 24, torch.float32, max_workspace_bytes=limit)
    gone = torch.zeros(700, dtype=torch.bool, device="cuda")
    gone[::5] = gone[1::5] = True
    a, b = (head.distill(h, w, index, s, temperature=2.0, token_scale=torch.where(gone, x, scale)) for x in (0.0, 1e38))
    for x, z in zip(a, b):
        assert torch.equal(x, z)
    each = [head.distill(h[t:t + 1], w, index[t:t + 1], s[t:t + 1], temperature=2.0) for t in (2, 3, 333, 699)]
    for t, r in zip((2, 3, 333, 699), each):
        assert (a.d_hidden[t] - scale[t] * r.d_hidden[0]).norm() <= 1e-5 * a.d_hidden[t].norm()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [30.0, 1e3, 1e5])
def test_certain_tokens(losses, dtype, size):
    """Tokens that are predicted with certainty, at logits of any size in range: the probability of the target does not exceed 1, so that no
    loss is below zero and no gradient points away from the target.  Every row of W but the target's is the target's turned round: then
    d_hidden = g (p_y - 1) 2 w_y, opposite to w_y or zero."""
    g = torch.Generator().manual_seed(3)
    row = torch.randn(200, generator=g)
    w = torch.stack([row, -row, -row, -row]).to(DT[dtype]).cuda()
    h = (row[None] * (size / float(row @ row)) * (0.3 + 0.7 * torch.rand(500, 1, generator=g))).to(DT[dtype]).cuda()
    h += torch.randn(500, 200, generator=g).to(DT[dtype]).cuda() * (size * 1e-3)
    y = torch.zeros(500, dtype=torch.int64, device="cuda")
    head = losses.LossHead(500, 4, 200, DT[dtype])
    s = torch.zeros(500, 1, device="cuda")
    for r in (head.cross_entropy(h, w, y), head.distill(h, w, y[:, None], s)):
        assert torch.isfinite(r.d_hidden).all() and torch.isfinite(r.d_weight).all()
        assert (r.loss >= 0).all() and (r.loss <= 1e-3 * max(size, 30.0)).all()
        assert (r.d_hidden.float() @ w[0].float() <= 0).all()

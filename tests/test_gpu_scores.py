"""Log probabilities, entropies, alternatives and their gradients through the HIP library against the fp64 oracle on the same inputs.

Tolerances.  A logit in the sums is an fp32 sum of D products: its error is below d = (4 + sqrt(D)) 2^-23 A with A = sum_d |h_d w_d| / tau, the
largest of the row.  lse carries d and a few roundings of its own size; log probabilities that and their own rounding, for their logits are
summed in double.  The entropy's derivative is -p (log p + entropy), whose magnitudes add up to 2 H at most: 2 H (d + 2^-20), 2^-20 for
the exponentials, plus 2^-20 (1 + H + log V) for the sums.  dz = g ([v = y] - p) - h p (log p + H): p carries 2 d (its logit's error and lse's),
log p + H that and the entropy's; bf16 rounds dz once, 2^-8 relative, and the result once more (2^-8); sums of K products add (8 + sqrt K) 2^-23 of their magnitudes.
Kept powers in f16 add 2^-11 of p and of log p, or half of f16's smallest step, 2^-40 of the largest of their block.
"""
import numpy as np
import pytest
import torch

from oracle import score_oracle as so
from tests.head_routes import ROUTES

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def losses():
    from paper_2502_16982_amd import losses as l
    return l


def as64(t):
    return None if t is None else t.detach().float().cpu().numpy().astype(np.float64)


def make(tokens, vocab, width, dtype, seed=0, pull=6.0):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(vocab, width, generator=g) * 0.05
    y = torch.randint(vocab, (tokens,), generator=g)
    h = torch.randn(tokens, width, generator=g)
    h += torch.rand(tokens, 1, generator=g) * pull * w[y] / (0.05 ** 2 * width)
    return h.to(DT[dtype]).cuda(), w.to(DT[dtype]).cuda(), y.cuda(), g


def errors(h64, w64, tau, lse, entropy):
    """(logit's, lse's, entropy's) per token."""
    live = np.isfinite(h64).all(axis=1)
    mag = np.abs(np.where(live[:, None], h64, 0.0)) @ np.abs(np.where(np.isfinite(w64), w64, 0.0)).T
    d = (4 + np.sqrt(h64.shape[1])) * 2.0 ** -23 * mag.max(axis=1) / tau + 2.0 ** -21
    big = np.nan_to_num(entropy)
    return d, d + 2.0 ** -22 * np.abs(np.nan_to_num(lse)), 2 * big * (d + 2.0 ** -20) + 2.0 ** -20 * (1 + big + np.log(w64.shape[0]))


def check(s, h, w, y, top=0, tau=1.0, live=None):
    h64, w64 = as64(h), as64(w)
    want = so.scores(h64, w64, None if y is None else y.cpu().numpy(), top, tau)
    live = np.isfinite(h64).all(axis=1) if live is None else live
    d, lse_err, h_err = errors(h64, w64, tau, want["lse"], want["entropy"])
    assert (np.abs(as64(s.lse) - want["lse"])[live] <= lse_err[live]).all()
    assert (np.abs(as64(s.entropy) - want["entropy"])[live] <= (h_err + 2.0 ** -23 * want["entropy"])[live]).all()
    assert (as64(s.entropy)[live] >= 0).all()
    if y is not None:
        lp = as64(s.log_prob)
        assert np.array_equal(np.isnan(lp)[live], np.isnan(want["log_prob"])[live])
        ok = live & ~np.isnan(want["log_prob"])
        assert (np.abs(lp - want["log_prob"])[ok] <= (lse_err + 2.0 ** -22 * np.abs(want["log_prob"]))[ok]).all()
        assert (lp[ok] <= 0).all()
    if top:
        assert np.array_equal(s.top_index.cpu().numpy()[live], want["top_index"][live])
        got, ref = as64(s.top_log_prob)[live], want["top_log_prob"][live]
        assert (got <= 0).all() and (np.abs(got - ref) <= lse_err[live][:, None] + 2.0 ** -22 * np.abs(ref)).all()
    return want


def results(s):
    return [t for t in s[:6] if t is not None]


def check_backward(grads, s, h, w, y, dl, de, tau=1.0, dtype="bf16"):
    h64, w64 = as64(h), as64(w)
    dl64, de64 = as64(dl), as64(de)
    want = so.scores(h64, w64, None if y is None else y.cpu().numpy(), 0, tau, dl64, de64)
    d, _, h_err = errors(h64, w64, tau, want["lse"], want["entropy"])
    tokens, vocab = len(h64), len(w64)
    yy = np.full(tokens, -1) if y is None else y.cpu().numpy()
    g = np.where((yy >= 0) & (yy < vocab), 0.0 if dl64 is None else dl64, 0.0)
    e = np.zeros(tokens) if de64 is None else de64
    kept = (g != 0) | (e != 0)
    with np.errstate(all="ignore"):
        logp = h64 @ w64.T / tau - want["lse"][:, None]
        p = np.exp(logp)
        bend = np.where(p == 0, 0.0, p * np.abs(logp + want["entropy"][:, None]))
    p, bend = np.where(kept[:, None], p, 0.0), np.where(kept[:, None], bend, 0.0)
    dz, g, e = np.abs(want["d_logits"]), np.abs(g)[:, None], np.abs(e)[:, None]
    spread = dz + 2 * g * p + 2 * e * bend                                 # where its parts cancel, their errors stay
    loose = spread * 2 * d[:, None] + e * p * (2 * d + np.nan_to_num(h_err))[:, None]
    if s.kept is not None and dtype == "bf16":
        loose = loose + (spread + e * p) * 2.0 ** -11 + (g + 64 * e) * 2.0 ** -39 * kept[:, None]
    h0 = np.where(kept[:, None], h64, 0.0)
    for got, ref, left, b, k in ((grads[0], want["d_hidden"], True, np.abs(w64), vocab), (grads[1], want["d_weight"], False, np.abs(h0), tokens)):
        if got is None:
            continue
        got = as64(got)
        assert np.isfinite(got).all()
        err = loose + spread * (8 + np.sqrt(k)) * 2.0 ** -23 + (dz * 2.0 ** -8 if dtype == "bf16" else 0.0)
        bound = (err @ b if left else err.T @ b) / tau + np.abs(ref) * (2.0 ** -7.99 if dtype == "bf16" else 2.0 ** -23) + 1e-37
        assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)
        noise = np.linalg.norm((loose @ b if left else loose.T @ b) / tau)
        assert np.linalg.norm(got - ref) <= (5e-3 if dtype == "bf16" else 1e-5) * np.linalg.norm(ref) + noise


SIZES = [(1, 1, 1, 1), (1, 7, 8, 7), (3, 129, 24, 2), (17, 1000, 64, 5), (64, 511, 136, 64), (65, 257, 33, 8), (130, 1027, 100, 0), (257, 130, 256, 3),
         (300, 2050, 520, 16), (2, 64, 16, 64), (5, 72, 40, 64), (9, 4099, 16, 33)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_sizes(losses, sizes, dtype):
    tokens, vocab, width, top = sizes
    h, w, y, g = make(tokens, vocab, width, dtype)
    y = torch.where(torch.rand(tokens, generator=g).cuda() < 0.2, -1, y)
    dl, de = torch.randn(tokens, generator=g).cuda(), torch.randn(tokens, generator=g).cuda() * 0.3
    for tau in (1.0, 0.7):
        head = losses.LossHead(tokens, vocab, width, DT[dtype])
        s = head.log_probs(h, w, y, top=top, temperature=tau)
        check(s, h, w, y, top, tau)
        check_backward(head.log_probs_backward(h, w, y, s, dl, de, temperature=tau), s, h, w, y, dl, de, tau, dtype)
        for keep in (True, False):
            s = head.log_probs(h, w, y, temperature=tau, keep=keep)
            assert (s.kept is not None) == (keep and (tokens > 64 or (dtype == "bf16" and (tokens > 16 or width % 8 == 0))))
            check(s, h, w, y, 0, tau)
            first = head.log_probs_backward(h, w, y, s, dl, de, temperature=tau)
            check_backward(first, s, h, w, y, dl, de, tau, dtype)
            for a, b in zip(first, head.log_probs_backward(h, w, y, s, dl, de, temperature=tau)):       # what is kept stays
                assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forms(losses, dtype):
    """int32 targets, none, one gradient alone, indexes beyond the vocabulary, no entropy's gradient, neither's."""
    h, w, y, g = make(70, 700, 96, dtype)
    head = losses.LossHead(70, 700, 96, DT[dtype])
    dl, de = torch.randn(70, generator=g).cuda(), torch.randn(70, generator=g).cuda()
    y[3], y[4], y[5] = -100, 700, 1 << 40
    s = head.log_probs(h, w, y, top=3)
    want = check(s, h, w, y, 3)
    assert np.isnan(want["log_prob"][4:6]).all() and float(s.log_prob[3]) == 0.0
    small = torch.where(y > 2 ** 31 - 1, 2 ** 31 - 1, y).to(torch.int32)
    again = head.log_probs(h, w, small, top=3)
    assert all(torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0)) for a, b in zip(results(s), results(again)))
    none = head.log_probs(h, w)
    assert none.log_prob is None and none.top_index is None and (none.entropy - s.entropy).abs().max() <= 1e-5 and (none.lse - s.lse).abs().max() <= 1e-5
    bare = head.log_probs(h, w, keep=False)
    assert torch.equal(bare.entropy, s.entropy) and torch.equal(bare.lse, s.lse)
    both = head.log_probs_backward(h, w, y, s, dl, de)
    check_backward(both, s, h, w, y, dl, de, 1.0, dtype)
    dh, nothing = head.log_probs_backward(h, w, y, s, dl, de, gradients=("hidden",))
    assert nothing is None and torch.equal(dh, both[0])
    nothing, dw = head.log_probs_backward(h, w, small, s, dl, de, gradients=("weight",))
    assert nothing is None and torch.equal(dw, both[1])
    check_backward(head.log_probs_backward(h, w, y, s, dl), s, h, w, y, dl, None, 1.0, dtype)
    check_backward(head.log_probs_backward(h, w, None, s, None, de), s, h, w, None, None, de, 1.0, dtype)
    zero = head.log_probs_backward(h, w, y, s, torch.zeros_like(dl))
    assert (zero[0] == 0).all() and (zero[1] == 0).all()
    assert head.log_probs_backward(h, w, y, s, dl, de, gradients=False) == (None, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties(losses, dtype):
    """Equal logits go by index: rows of zeros, weight rows that come twice, all of them alike."""
    h, w, y, _ = make(40, 5000, 64, dtype)
    h[7] = 0
    w[1000:2000] = w[:1000]
    w[4000] = w[999]
    head = losses.LossHead(40, 5000, 64, DT[dtype])
    for top in (1, 8, 50):
        s = head.log_probs(h, w, y, top=top)
        assert s.top_index[7].tolist() == list(range(top))
        if dtype == "bf16":                                                # sums of products of bf16 in double are exact here
            check(s, h, w, y, top)
    w[:] = w[5]
    s = head.log_probs(h, w, y, top=20)
    assert (s.top_index == torch.arange(20, device="cuda")).all()
    assert ((s.entropy - np.log(5000)).abs() <= 2.0 ** -19 * 10).all() and ((s.log_prob + np.log(5000)).abs() <= 2.0 ** -19 * 10).all()


def test_alternatives_that_lie_together(losses):
    """The largest logits in neighbouring entries, whose groups have to be looked through."""
    h, w, y, g = make(33, 3000, 64, "bf16")
    for t in range(33):
        at = (t * 89) % 2900
        w[at:at + 40] = (h[t].float() * (0.2 + 0.002 * torch.randperm(40, generator=g).cuda()[:, None])).to(torch.bfloat16)
    head = losses.LossHead(33, 3000, 64)
    for top in (1, 5, 32, 64):
        check(head.log_probs(h, w, y, top=top), h, w, y, top)


def test_alternatives_that_few_threads_hold(losses):
    """More groups above what the threads' own largest bound than the list holds: 71 of each 256 groups, 64 times."""
    vocab, width = 1 << 19, 8
    row = torch.arange(vocab)
    group = row // 64 * 2 + row // 4 % 2
    g = torch.Generator().manual_seed(5)
    value = torch.rand(vocab, generator=g) + 3.0 * (group % 256 < 71)
    w = torch.zeros(vocab, width)
    w[:, 0] = value
    h = torch.zeros(3, width)
    h[:, 0] = torch.tensor([1.0, 2.0, -1.0])
    head = losses.LossHead(3, vocab, width, torch.float32)
    s = head.log_probs(h.cuda(), w.cuda(), None, top=64)
    order = value.double().sort(descending=True, stable=True).indices
    assert torch.equal(s.top_index[0].cpu(), order[:64]) and torch.equal(s.top_index[1].cpu(), order[:64])
    assert torch.equal(s.top_index[2].cpu(), value.double().sort(stable=True).indices[:64])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite(losses, dtype):
    """A token's hidden state that is NaN: its own results only, and no gradient of the weight unless it has one itself."""
    h, w, y, g = make(50, 900, 72, dtype)
    bad = h.clone()
    bad[11], bad[30, 5], bad[49, 71] = float("nan"), float("inf"), float("nan")
    rows = [11, 30, 49]
    keep = np.ones(50, dtype=bool)
    keep[rows] = False
    head = losses.LossHead(50, 900, 72, DT[dtype])
    s, clean = head.log_probs(bad, w, y, top=5), head.log_probs(h, w, y, top=5)
    check(s, bad, w, y, 5, live=keep)
    for a, b in zip(results(s), results(clean)):
        assert torch.equal(a[torch.from_numpy(keep).cuda()], b[torch.from_numpy(keep).cuda()])
    assert s.lse[11].isnan() and s.log_prob[11].isnan() and s.entropy[11].isnan()
    assert ((s.top_index >= 0) & (s.top_index < 900)).all()
    dl, de = torch.randn(50, generator=g).cuda(), torch.randn(50, generator=g).cuda()
    dl[rows], de[rows] = 0.0, 0.0
    dh, dw = head.log_probs_backward(bad, w, y, s, dl, de)
    want = head.log_probs_backward(h, w, y, clean, dl, de)
    assert torch.equal(dw, want[1]) and torch.equal(dh, want[0]) and (dh[rows] == 0).all()
    s, clean = head.log_probs(bad, w, y), head.log_probs(h, w, y)
    dh, dw = head.log_probs_backward(bad, w, y, s, dl, de)
    want = head.log_probs_backward(h, w, y, clean, dl, de)
    assert (s.kept is not None) == (dtype == "bf16") and torch.equal(dw, want[1]) and torch.equal(dh, want[0]) and (dh[rows] == 0).all()


def test_logits_of_minus_infinity(losses):
    """Masked vocabulary entries: weights so low that their logits are -inf, whole blocks of them and single ones."""
    h, w, y, g = make(20, 1500, 16, "f32")
    h[:, 0], w[:, 0] = 2.0, 0.0
    w[128:512, 0], w[700, 0], w[1499, 0] = -3e38, -3e38, -3e38
    y = torch.where((y >= 128) & (y < 512), 5, y)
    y[0] = 700
    head = losses.LossHead(20, 1500, 16, torch.float32)
    s = head.log_probs(h, w, y, top=64)
    z = h.double().cpu() @ w.double().cpu().T
    z[:, 128:512], z[:, 700], z[:, 1499] = -torch.inf, -torch.inf, -torch.inf
    logp = torch.log_softmax(z, 1)
    assert float(s.log_prob[0]) < -1e38 and not s.entropy.isnan().any()
    assert (s.log_prob[1:].double().cpu() - logp.gather(1, y.cpu()[:, None])[1:, 0]).abs().nan_to_num(0.0, 0.0, 0.0).max() <= 1e-5
    assert (s.entropy.double().cpu() - torch.special.entr(logp.exp()).sum(1)).abs().max() <= 1e-4
    assert torch.equal(s.top_index.cpu(), logp.topk(64).indices)
    y[0] = 3
    de = torch.ones(20, device="cuda")
    for keep in (True, False):
        s = head.log_probs(h, w, y, keep=keep)
        dh, dw = head.log_probs_backward(h, w, y, s, de, de)
        assert not dw.isnan().any() and (dw[128:512] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", ROUTES)
def test_every_form_of_launch(losses, tokens, vocab, width, dtype):
    """Sizes that take each form of tile, against 64 bits on the GPU."""
    h, w, y, g = make(tokens, vocab, width, dtype, pull=9.0)
    dl, de = torch.randn(tokens, generator=g).cuda() / tokens, torch.full((tokens,), 0.1 / tokens, device="cuda")
    head = losses.LossHead(tokens, vocab, width, DT[dtype])
    s = head.log_probs(h, w, y, top=4, temperature=1.3)
    dh, dw = head.log_probs_backward(h, w, y, s, dl, de, temperature=1.3)
    k = head.log_probs(h, w, y, temperature=1.3)
    dh2, dw2 = head.log_probs_backward(h, w, y, k, dl, de, temperature=1.3)
    assert k.kept is not None or (tokens <= 64 and (dtype == "f32" or width % 8))
    logp = torch.log_softmax(h.double() @ w.double().T.contiguous() / 1.3, 1)
    entropy = torch.special.entr(logp.exp()).sum(1)
    best = logp.topk(4)
    assert torch.equal(s.top_index, best.indices)
    for got, want in ((s.log_prob, logp.gather(1, y[:, None])[:, 0]), (s.entropy, entropy), (s.top_log_prob, best.values), (k.log_prob, logp.gather(1, y[:, None])[:, 0]),
                      (k.entropy, entropy)):
        assert (got.double() - want).norm() <= 2e-6 * want.norm()
    p = logp.exp()
    dz = -p * (dl.double()[:, None] + de.double()[:, None] * (logp + entropy[:, None]))
    dz[torch.arange(tokens), y] += dl.double()
    dh64, dw64 = dz @ w.double() / 1.3, dz.T.contiguous() @ h.double() / 1.3
    for got, want in ((dh, dh64), (dw, dw64), (dh2, dh64), (dw2, dw64)):
        assert (got.double() - want).norm() <= (5e-3 if dtype == "bf16" else 1e-5) * want.norm()


@pytest.mark.parametrize("dtype,tokens", [("bf16", 1), ("bf16", 16), ("bf16", 17), ("f32", 1), ("f32", 16), ("f32", 17), ("f32", 33), ("f32", 64), ("f32", 65)])
@pytest.mark.parametrize("vocab,width", [(1, 1), (127, 3), (129, 31), (1000, 65), (700, 515), (4100, 129)])
def test_few_tokens(losses, dtype, tokens, vocab, width):
    """Rows as they are, of odd widths and, in a wider buffer, at odd addresses; on both sides of the limits."""
    h, w, y, g = make(tokens, vocab, width, dtype, seed=tokens)
    y = torch.where(torch.rand(tokens, generator=g).cuda() < 0.2, -1, y)
    head = losses.LossHead(tokens, vocab, width, DT[dtype], gradients=False)
    top = min(vocab, 9)
    s = head.log_probs(h, w, y, top=top, temperature=0.8)
    check(s, h, w, y, top, 0.8)
    bare = head.log_probs(h, w, y, temperature=0.8)
    assert all(torch.equal(a, b) for a, b in zip(results(s)[:4], results(bare)))
    rows, tall = torch.full((tokens, width + 5), 9.0, dtype=DT[dtype], device="cuda"), torch.full((vocab, width + 7), 9.0, dtype=DT[dtype], device="cuda")
    rows[:, 1:1 + width], tall[:, 3:3 + width] = h, w
    for a, b in zip(results(s), results(head.log_probs(rows[:, 1:1 + width], tall[:, 3:3 + width], y, top=top, temperature=0.8))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pieces(losses, dtype):
    """A limited workspace gives the same scores, in pieces of tokens; the weight's gradient is summed over them in fp32."""
    h, w, y, g = make(1000, 1300, 80, dtype)
    whole = losses.LossHead(1000, 1300, 80, DT[dtype])
    few = losses.LossHead(1000, 1300, 80, DT[dtype], max_workspace_bytes=1)
    a, b = whole.log_probs(h, w, y, top=6), few.log_probs(h, w, y, top=6)
    check(b, h, w, y, 6)
    assert torch.equal(a.top_index, b.top_index)
    dl, de = torch.randn(1000, generator=g).cuda(), torch.randn(1000, generator=g).cuda()
    check_backward(few.log_probs_backward(h, w, y, b, dl, de), b, h, w, y, dl, de, 1.0, dtype)
    assert few.workspace.numel() < whole.workspace.numel()
    b = few.log_probs(h, w, y)
    assert b.kept is None
    b = few.log_probs(h, w, y, keep=True)
    check(b, h, w, y)
    check_backward(few.log_probs_backward(h, w, y, b, dl, de), b, h, w, y, dl, de, 1.0, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_alignment(losses, dtype):
    h, w, y, g = make(60, 500, 64, dtype)
    wide, tall = torch.zeros(60, 101, dtype=DT[dtype], device="cuda"), torch.zeros(500, 99, dtype=DT[dtype], device="cuda")
    wide[:, 3:67], tall[:, 1:65] = h, w
    head = losses.LossHead(60, 500, 64, DT[dtype])
    dl = torch.randn(60, generator=g).cuda()
    a, b = head.log_probs(h, w, y, top=4), head.log_probs(wide[:, 3:67], tall[:, 1:65], y, top=4)
    assert all(torch.equal(x, z) for x, z in zip(results(a), results(b)))
    for x, z in zip(head.log_probs_backward(h, w, y, a, dl, dl), head.log_probs_backward(wide[:, 3:67], tall[:, 1:65], y, b, dl, dl)):
        assert torch.equal(x, z)


def test_beside_the_losses(losses):
    """One LossHead for cross entropy, scores and their gradients in turn; the log probabilities are minus its loss, its gradients those of it."""
    h, w, y, g = make(200, 3000, 128, "bf16")
    y[::7] = -1
    head = losses.LossHead(200, 3000, 128)
    scale = torch.rand(200, generator=g).cuda()
    ce = head.cross_entropy(h, w, y, token_scale=scale)
    s = head.log_probs(h, w, y, top=2)
    again = head.cross_entropy(h, w, y, token_scale=scale)
    dh, dw = head.log_probs_backward(h, w, y, s, -scale)
    assert torch.equal(ce.d_weight, again.d_weight) and torch.equal(ce.loss, again.loss)
    assert (ce.loss + s.log_prob).abs().max() <= 1e-5 and (ce.lse - s.lse).abs().max() <= 1e-5
    for a, b in ((dh, ce.d_hidden), (dw, ce.d_weight)):
        assert (a.float() - b.float()).norm() <= 5e-3 * b.float().norm()


def test_streams_and_capture(losses):
    h, w, y, g = make(90, 2100, 96, "bf16")
    dl, de = torch.randn(90, generator=g).cuda(), torch.randn(90, generator=g).cuda()
    head = losses.LossHead(90, 2100, 96)

    def both(h, y):
        s, k = head.log_probs(h, w, y, top=5), head.log_probs(h, w, y)
        return [*results(s), *results(k), *head.log_probs_backward(h, w, y, s, dl, de), *head.log_probs_backward(h, w, y, k, dl, de)]

    want = both(h, y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = both(h, y)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, there))
    hold_h, hold_y = h.clone(), y.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(hold_h, hold_y)
    for seed in range(3):
        h2, _, y2, _ = make(90, 2100, 96, "bf16", seed=20 + seed)
        hold_h.copy_(h2)
        hold_y.copy_(y2)
        eager = both(h2, y2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))


def test_no_tokens(losses):
    h, w, y, _ = make(4, 300, 32, "bf16")
    head = losses.LossHead(4, 300, 32)
    s = head.log_probs(h[:0], w, y[:0], top=3)
    assert s.log_prob.shape == (0,) and s.top_index.shape == (0, 3)
    for s in (s, head.log_probs(h[:0], w, y[:0])):
        dh, dw = head.log_probs_backward(h[:0], w, y[:0], s, s.log_prob)
        assert dh.shape == (0, 32) and (dw == 0).all()


def test_gradients_from_rows_of_another_alignment(losses):
    """Scores that kept their powers, gradients by the same values in rows that would be copied: the logits are made again."""
    h, w, y, g = make(5, 700, 64, "bf16")
    head = losses.LossHead(5, 700, 64)
    s = head.log_probs(h, w, y)
    assert s.kept is not None
    dl, de = torch.randn(5, generator=g).cuda(), torch.randn(5, generator=g).cuda()
    other = torch.empty(700 * 64 + 1, dtype=w.dtype, device="cuda")[1:].view(700, 64).copy_(w)
    check_backward(head.log_probs_backward(h, other, y, s, dl, de), s, h, w, y, dl, de)
    check_backward(head.log_probs_backward(h, w, y, head.log_probs(h, other, y), dl, de), s, h, w, y, dl, de)


@pytest.mark.parametrize("dtype,tokens,vocab,width", [("f32", 3, 70001, 32768), ("bf16", 24, 140001, 32768), ("bf16", 5, 280001, 16385)])
def test_weights_beyond_32_bits(losses, dtype, tokens, vocab, width):
    """The weight's last rows, the only ones that are not zero, start beyond 2^31 elements (fp32: 2^32 bytes)."""
    last = 300
    g = torch.Generator().manual_seed(3)
    few = (torch.randn(last, width, generator=g) * 0.02).to(DT[dtype]).cuda()
    w = torch.zeros(vocab, width, dtype=DT[dtype], device="cuda")
    w[-last:] = few
    h = torch.randn(tokens, width, generator=g).to(DT[dtype]).cuda()
    y = torch.randint(vocab - last, vocab, (tokens,), generator=g).cuda()
    head = losses.LossHead(tokens, vocab, width, DT[dtype], gradients=False)
    s = head.log_probs(h, w, y, top=2)
    h64, w64 = as64(h), as64(few)
    z = h64 @ w64.T
    lse = np.log(vocab - last + np.exp(z).sum(axis=1))
    entropy = lse - (np.exp(z - lse[:, None]) * z).sum(axis=1)
    _, lse_err, h_err = errors(h64, w64, 1.0, lse, entropy)
    h_err = h_err + 2.0 ** -20 * np.log(vocab)
    order = np.argsort(-z, axis=1)[:, :2]
    assert (np.abs(as64(s.lse) - lse) <= lse_err).all()
    assert (np.abs(as64(s.entropy) - entropy) <= h_err).all()
    assert np.array_equal(s.top_index.cpu().numpy(), order + vocab - last)
    for got, at in ((s.log_prob[:, None], (y.cpu().numpy() - vocab + last)[:, None]), (s.top_log_prob, order)):
        want = np.take_along_axis(z, at, 1) - lse[:, None]
        assert (np.abs(as64(got) - want) <= lse_err[:, None] + 2.0 ** -22 * np.abs(want)).all()


def test_kept_powers_beyond_32_bits(losses):
    """17000 x 131072 kept powers; the last tokens are the only ones with gradients."""
    tokens, vocab, width, last = 17000, 131072, 64, 48
    h, w, y, g = make(tokens, vocab, width, "bf16")
    dl, de = torch.zeros(tokens), torch.zeros(tokens)
    dl[-last:], de[-last:] = torch.randn(last, generator=g), torch.randn(last, generator=g) * 0.3
    dl, de = dl.cuda(), de.cuda()
    head = losses.LossHead(tokens, vocab, width)
    s = head.log_probs(h, w, y)
    assert s.kept.numel() > 2 ** 32
    dh, dw = head.log_probs_backward(h, w, y, s, dl, de)
    assert (dh[:-last] == 0).all()
    part = losses.TokenScores(*(None if t is None else t[-last:] for t in s[:6]), s.kept)
    check(part, h[-last:], w, y[-last:])
    check_backward((dh[-last:], dw), part, h[-last:], w, y[-last:], dl[-last:], de[-last:])


@pytest.mark.parametrize("tokens,vocab,width", [(64, 1024, 64), (171, 36393, 72)])
def test_entropy_of_peaked_rows(losses, tokens, vocab, width):
    """A token's likeliest entry and n others in one block, everything else without weight, logits exact (hidden states pick a column of the weight).

    With a_i = z_top - z_i, q the probabilities, A = sum q a, rounding steps u = 2^-24: sums of n + 1 powers and of their products with exponents, and
    two joins of waves, are off by (n + 2) u of themselves, a power by 2 u (the instruction's last bit) and by a_i u (its exponent's rounding), the products by u, the
    exponents' unit by u.  entropy = log S + A takes an error e of a power i with q_i e (1 + a_i + A) and one of S with (1 + A); the result is rounded once more.
    Exponents relative to anything but the largest would carry steps of their own size."""
    g = torch.Generator().manual_seed(0)
    z = torch.full((vocab, width), -200.0)
    top = (torch.rand(width, generator=g) * 16 - 8).bfloat16().float()
    for c in range(width):
        n = 1 + c % 4
        at = int(torch.randint(vocab // 128, (1,), generator=g)) * 128 + torch.randperm(128, generator=g)[:n + 1]
        z[at[0], c] = top[c]
        z[at[1:], c] = (top[c] - 0.5 - c // 4 * 0.85 - torch.rand(n, generator=g)).bfloat16().float()
    h = torch.eye(width)[torch.arange(tokens) % width].bfloat16().cuda()
    head = losses.LossHead(tokens, vocab, width)
    z64 = z.double().numpy().T[np.arange(tokens) % width]
    a = z64.max(1, keepdims=True) - z64
    p = np.where(a < 100, np.exp(-a), 0.0)
    lse = z64.max(1) + np.log(p.sum(1))
    q, n = p / p.sum(1, keepdims=True), (p > 0).sum(1) - 1
    a = np.where(p > 0, a, 0.0)
    mean = (q * a).sum(1)
    entropy = np.log(p.sum(1)) + mean
    others = np.where(a > 0, q, 0.0) * (2 + a)
    err = 2.0 ** -24 * ((n + 2) * (1 + 2 * mean) + 2 * (1 + mean) + mean + (others * (1 + a + mean[:, None])).sum(1) + (q * a * a).sum(1))
    lse_err = 2.0 ** -24 * (n + 4 + others.sum(1) + mean)
    for s in (head.log_probs(h, z.bfloat16().cuda(), keep=True), head.log_probs(h, z.bfloat16().cuda(), keep=False), head.log_probs(h, z.bfloat16().cuda(), top=3)):
        assert (np.abs(as64(s.entropy) - entropy) <= err + 2.0 ** -24 * entropy).all(), np.max(np.abs(as64(s.entropy) - entropy) / err)
        assert (np.abs(as64(s.lse) + as64(s.lse_rest) - lse) <= lse_err + 2.0 ** -48 * np.abs(lse)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_logits_that_are_not_finite(losses, dtype):
    """A token with gradients whose logits are NaN or infinite: no gradient of its own and none of the weight is finite; the other tokens' rows stay."""
    h, w, y, g = make(90, 900, 72, dtype)
    dl, de = torch.randn(90, generator=g).cuda(), torch.randn(90, generator=g).cuda()
    head = losses.LossHead(90, 900, 72, DT[dtype])
    for value in (float("nan"), float("inf")):
        bad = h.clone()
        bad[11, 5] = value
        rest = [t for t in range(90) if t != 11]
        for keep in (True, False):
            s, clean = head.log_probs(bad, w, y, keep=keep), head.log_probs(h, w, y, keep=keep)
            for a, b, to in ((dl, None, y), (dl, de, y), (None, de, None)):
                dh, dw = head.log_probs_backward(bad, w, to, s, a, b)
                want, _ = head.log_probs_backward(h, w, to, clean, a, b)
                assert dh[11].isnan().all() and torch.equal(dh[rest], want[rest])
                assert dw.isnan().all(), (value, keep, a is None, b is None, int(dw.isnan().all(1).sum()))


def test_long_batches_keep_nothing_by_default(losses):
    """36000 x 131072: powers would take more than is kept unasked for; the logits are made again."""
    tokens, vocab, width, last = 36000, 131072, 64, 48
    h, w, y, g = make(tokens, vocab, width, "bf16")
    dl, de = torch.zeros(tokens), torch.zeros(tokens)
    dl[-last:], de[-last:] = torch.randn(last, generator=g), torch.randn(last, generator=g) * 0.3
    dl, de = dl.cuda(), de.cuda()
    head = losses.LossHead(tokens, vocab, width)
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    s = head.log_probs(h, w, y)
    assert s.kept is None and torch.cuda.max_memory_allocated() - before < 2 ** 24
    dh, dw = head.log_probs_backward(h, w, y, s, dl, de)
    assert (dh[:-last] == 0).all()
    part = losses.TokenScores(*(None if t is None else t[-last:] for t in s[:6]))
    check(part, h[-last:], w, y[-last:])
    check_backward((dh[-last:], dw), part, h[-last:], w, y[-last:], dl[-last:], de[-last:])


@pytest.mark.parametrize("dtype,tokens", [("bf16", 16), ("bf16", 17), ("f32", 64), ("f32", 65)])
def test_alternatives_that_fp32_cannot_tell_apart(losses, dtype, tokens):
    """Twelve entries in groups of their own whose logits differ by less than fp32 sums resolve, more than are picked beside the asked for, on both sides of
    the limits of few tokens: what comes back is within the sums' error of the largest, and in the order of sums in double."""
    vocab, width, top = 3000, 515, 3
    h, w, y, g = make(tokens, vocab, width, dtype, pull=0.0)
    row, at = torch.randn(width, generator=g).to(DT[dtype]).cuda() * 0.5, torch.arange(12, device="cuda") * 224 + 5
    h = (h.float() * 0.1 + row.float()).to(DT[dtype])
    w[at] = row
    h[:, 0], w[:, 0] = 2.0 ** -20, 0.0
    w[at, 0] = torch.randperm(12, generator=g).to(DT[dtype]).cuda() + 1
    head = losses.LossHead(tokens, vocab, width, DT[dtype], gradients=False)
    s = head.log_probs(h, w, top=top)
    h64, w64 = as64(h), as64(w)
    want = so.scores(h64, w64, None, 12)
    d, lse_err, _ = errors(h64, w64, 1.0, want["lse"], want["entropy"])
    z, index = h64 @ w64.T, s.top_index.cpu().numpy()
    got = np.take_along_axis(z, index, 1)
    assert np.isin(index, at.cpu().numpy()).all() and all(len(set(i)) == top for i in index)
    assert (np.sort(z, axis=1)[:, -12] - np.sort(z, axis=1)[:, -13] > 2 * d).all() and (np.ptp(np.sort(z, axis=1)[:, -12:], axis=1) < d).all()
    assert (got >= want["top_log_prob"][:, top - 1:top] + want["lse"][:, None] - 2 * d[:, None]).all()
    assert (np.diff(got, axis=1) < 0).all()
    assert (np.abs(as64(s.top_log_prob) - (got - want["lse"][:, None])) <= lse_err[:, None] + 2.0 ** -22 * np.abs(got - want["lse"][:, None])).all()

"""The head's losses and their gradients through the HIP library against the fp64 oracle on the same inputs.

Tolerances.  A logit is an fp32 sum of D products: its error is below (4 + sqrt(D)) 2^-23 A with A = sum_d |h_d w_d| / tau (rounding
errors of the sum average; the worst case, D 2^-24 A, is never near).  lse carries the largest such error of its row plus a few
roundings of its own size; the loss carries two.  In fp32 a gradient's error is that of dz (relative: the error of the logits) and that
of a sum of K products of three-plane operands, both relative to the sum of magnitudes |dz| |W|.  In bf16 dz is rounded once, at most
2^-8 relative (8 bits of significand), on top of f16's 2^-11 for the probabilities (or half of f16's smallest step, 2^-39 of the largest of
their block), and the result once more: at most 2^-7.8 of the sum of
magnitudes plus 2^-8 of the result; as a whole (2-norm) each of the two contributes about 1.7e-3, together 2.4e-3: held to 5e-3.
"""
import numpy as np
import pytest
import torch

from oracle import head_oracle as ho
from tests.head_routes import ROUTES

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def losses():
    from paper_2502_16982_amd import losses as l
    return l


def as64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def make(tokens, vocab, width, dtype, seed=0, pull=6.0):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(vocab, width, generator=g) * 0.05
    y = torch.randint(vocab, (tokens,), generator=g)
    h = torch.randn(tokens, width, generator=g)
    h += torch.rand(tokens, 1, generator=g) * pull * w[y] / (0.05 ** 2 * width)
    return h.to(DT[dtype]).cuda(), w.to(DT[dtype]).cuda(), y.cuda(), g


def make_teacher(tokens, vocab, top, g):
    index = torch.stack([torch.randperm(vocab, generator=g)[:top] for _ in range(tokens)]) if top <= vocab else torch.randint(vocab, (tokens, top), generator=g)
    return index, torch.randn(tokens, top, generator=g) * 2


def check(r, h, w, dtype, tau=1.0, scale=None, **target):
    h64, w64 = as64(h), as64(w)
    want = ho.head_loss(h64, w64, tau=tau, scale=None if scale is None else as64(scale), **target)
    width, vocab = h64.shape[1], w64.shape[0]
    live = np.isfinite(h64).all(axis=1)
    mag = np.abs(np.where(live[:, None], h64, 0.0)) @ np.abs(w64).T
    dz_err = (4 + np.sqrt(width)) * 2.0 ** -23 * mag.max(axis=1) / tau + 2.0 ** -21
    lse_err = dz_err + 2.0 ** -22 * np.abs(np.where(live, want["lse"], 0.0))
    if r.lse is not None:
        lse = as64(r.lse)
        assert (np.abs(lse - want["lse"])[live] <= lse_err[live]).all()
    loss = as64(r.loss)
    assert np.array_equal(np.isnan(loss), np.isnan(want["loss"]))
    s = 0.0 if "teacher" not in target else np.abs(np.nan_to_num(target["teacher"], nan=0.0, neginf=0.0)).max() / tau
    ok = ~np.isnan(loss) & live
    assert (np.abs(loss - want["loss"])[ok] <= (tau * tau * (2 * lse_err + 2.0 ** -22 * s) + 2.0 ** -23 * np.abs(want["loss"]))[ok]).all()
    assert (loss[~live & ~np.isnan(want["loss"])] == 0.0).all()
    dz = np.abs(want["d_logits"])
    g = np.ones(len(loss)) if scale is None else np.abs(as64(scale))
    if "targets" in target:
        kept = (g != 0) & (target["targets"] >= 0) & (target["targets"] < vocab)
    else:
        kept = (g != 0) & ((target["index"] >= 0) & ~np.isneginf(target["teacher"])).any(1) & (target["index"] < vocab).all(1)
    with np.errstate(all="ignore"):
        p = np.where(kept[:, None], np.exp(h64 @ w64.T / tau - want["lse"][:, None]), 0.0)
    spread = dz + 2 * tau * g[:, None] * p                                 # |dz| <= g tau (p + q): where they cancel, p's error stays
    h0 = np.where(kept[:, None], h64, 0.0)
    for got, ref, a, b, k in ((r.d_hidden, want["d_hidden"], np.eye(len(loss)), np.abs(w64), vocab),
                              (r.d_weight, want["d_weight"], None, np.abs(h0), len(loss))):
        if got is None:
            continue
        got = as64(got)
        assert np.isfinite(got).all()
        if dtype == "f32":
            e = spread * (2 * dz_err[:, None] + (8 + np.sqrt(k)) * 2.0 ** -23)
        else:
            e = dz * 2.0 ** -7.8 + spread * 2 * dz_err[:, None] + np.where(kept, tau * g * 2.0 ** -40, 0.0)[:, None]
        bound = (e @ b if a is not None else e.T @ b) + np.abs(ref) * (2.0 ** -7.99 if dtype == "bf16" else 2.0 ** -23) + 1e-37
        assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)
        noise = spread * 2 * dz_err[:, None]                               # all there is of a gradient that cancels to nothing
        noise = np.linalg.norm(noise @ b if a is not None else noise.T @ b)
        assert np.linalg.norm(got - ref) <= (5e-3 if dtype == "bf16" else 1e-5) * np.linalg.norm(ref) + noise


SIZES = [(1, 1, 1), (1, 7, 8), (3, 129, 24), (17, 1000, 64), (64, 511, 136), (65, 257, 33), (130, 1027, 100), (257, 130, 256), (300, 2050, 520)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", SIZES)
def test_cross_entropy(losses, tokens, vocab, width, dtype):
    h, w, y, g = make(tokens, vocab, width, dtype)
    gone = torch.rand(tokens, generator=g) < 0.2
    y = torch.where(gone.cuda(), -100, y)
    scale = torch.rand(tokens, generator=g).cuda() + 0.1
    head = losses.LossHead(tokens, vocab, width, DT[dtype])
    r = head.cross_entropy(h, w, y, token_scale=scale)
    check(r, h, w, dtype, scale=scale, targets=y.cpu().numpy())
    e = head.cross_entropy(h, w, y.to(torch.int32), gradients=False)
    assert e.d_hidden is None and e.d_weight is None
    check(e, h, w, dtype, targets=y.cpu().numpy())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", SIZES)
@pytest.mark.parametrize("top,tau", [(1, 1.0), (5, 2.0), (70, 0.7)])
def test_distill(losses, tokens, vocab, width, dtype, top, tau):
    h, w, _, g = make(tokens, vocab, width, dtype, seed=top)
    index, s = make_teacher(tokens, vocab, top, g)          # more entries than vocabulary: some twice
    none = torch.rand(tokens, top, generator=g)
    index[none < 0.15] = -1
    s[none < 0.1] = float("nan")                            # behind a negative index: never read as a number
    s[(none >= 0.15) & (none < 0.25)] = -float("inf")
    index[:1], s[:1] = torch.arange(top) % vocab, torch.arange(top) * 0.1
    if tokens > 2:
        index[2] = -1                                       # a token without entries
    scale = torch.rand(tokens, generator=g).cuda() + 0.1
    head = losses.LossHead(tokens, vocab, width, DT[dtype])
    r = head.distill(h, w, index.cuda(), s.cuda(), temperature=tau, token_scale=scale)
    check(r, h, w, dtype, tau=tau, scale=scale, index=index.numpy(), teacher=s.double().numpy())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", ROUTES)
def test_every_form_of_launch(losses, tokens, vocab, width, dtype):
    """Against the formulas in fp64 on the device (the oracle's rows one by one would take minutes), block by block of 64 x 64 of the
    gradients: a wrong or missing tile shows in its own block."""
    h, w, y, g = make(tokens, vocab, width, dtype)
    y[torch.rand(tokens, generator=g) < 0.1] = -100
    scale = (torch.rand(tokens, generator=g) + 0.5).cuda() / tokens
    r = losses.LossHead(tokens, vocab, width, DT[dtype]).cross_entropy(h, w, y, token_scale=scale)
    h64, w64, kept = h.double(), w.double(), y >= 0
    z = torch.mm(h64, w64.T.contiguous())
    lse = torch.logsumexp(z, 1)
    at = y.clamp(min=0)[:, None]
    loss = torch.where(kept, lse - z.gather(1, at)[:, 0], 0.0)
    err = (4 + width ** 0.5) * 2.0 ** -23 * torch.mm(h64.abs(), w64.abs().T.contiguous()).amax(1) + 2.0 ** -21 + 2.0 ** -22 * lse.abs()
    assert ((r.lse - lse).abs() <= err).all() and ((r.loss - loss).abs() <= 2 * err + 2.0 ** -23 * loss).all()
    dz = (z - lse[:, None]).exp()
    dz.scatter_add_(1, at, torch.full_like(loss, -1.0)[:, None])
    dz *= (scale.double() * kept)[:, None]
    for got, want in ((r.d_hidden, torch.mm(dz, w64)), (r.d_weight, torch.mm(dz.T.contiguous(), h64))):
        rows, cols = -(-got.shape[0] // 64) * 64, -(-got.shape[1] // 64) * 64
        blocks = []
        for x in (got.double() - want, want):
            full = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
            full[:x.shape[0], :x.shape[1]] = x
            blocks.append(full.view(rows // 64, 64, cols // 64, 64).square().sum((1, 3)).sqrt())
        # twice the bar of the whole in a block (fewer roundings average), and never held to less than a thousandth of the typical block
        bar = 2 * (5e-3 if dtype == "bf16" else 1e-5)
        assert (blocks[0] <= bar * blocks[1].clamp(min=1e-3 * float(blocks[1].square().mean().sqrt()))).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_tokens_may_hold_anything(losses, dtype):
    """Hidden states of ignored tokens, of tokens with scale 0 and of those with a target beyond the vocabulary reach no gradient."""
    h, w, y, _ = make(70, 300, 64, dtype)
    h[3], h[10], h[20], h[40] = float("nan"), float("inf"), -float("inf"), float("nan")
    y[3], y[10], y[20], y[40] = -100, -1, 5, 300
    scale = torch.ones(70, device="cuda")
    scale[20] = 0.0
    head = losses.LossHead(70, 300, 64, DT[dtype])
    r = head.cross_entropy(h, w, y, token_scale=scale)
    assert torch.isnan(r.loss[40]) and r.loss[3] == 0.0 and r.loss[10] == 0.0
    for t in (3, 10, 20, 40):
        assert not r.d_hidden[t].any()
    assert torch.isfinite(r.d_hidden).all() and torch.isfinite(r.d_weight).all()
    live = torch.ones(70, dtype=torch.bool, device="cuda")
    live[[3, 10, 20, 40]] = False
    part = losses.LossHead(70, 300, 64, DT[dtype]).cross_entropy(h[live], w, y[live])
    assert torch.equal(part.loss, r.loss[live]) and torch.equal(part.d_hidden, r.d_hidden[live])
    want = ho.head_loss(as64(h[live]), as64(w), targets=y[live].cpu().numpy())["d_weight"]
    assert np.linalg.norm(as64(r.d_weight) - want) <= (5e-3 if dtype == "bf16" else 1e-5) * np.linalg.norm(want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits(losses, dtype):
    """Logits of some hundreds: nothing overflows, near-certain tokens keep their small gradients."""
    h, w, y, _ = make(40, 500, 64, dtype)
    h = h * 40
    head = losses.LossHead(40, 500, 64, DT[dtype])
    check(head.cross_entropy(h, w, y), h, w, dtype, targets=y.cpu().numpy())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width,extra", [(64, 8), (64, 3), (50, 0), (40, 24)])
def test_strides_and_alignment(losses, dtype, width, extra):
    h, w, y, _ = make(70, 300, width, dtype)
    hs = torch.full((70, width + extra), float("nan"), dtype=DT[dtype], device="cuda")[:, extra // 2:extra // 2 + width]
    ws = torch.full((300, width + extra), float("nan"), dtype=DT[dtype], device="cuda")[:, extra // 2:extra // 2 + width]
    hs.copy_(h)
    ws.copy_(w)
    head = losses.LossHead(70, 300, width, DT[dtype])
    r = head.cross_entropy(hs, ws, y)
    check(r, h, w, dtype, targets=y.cpu().numpy())
    plain = head.cross_entropy(h, w, y)
    for a, b in zip(r, plain):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pieces_of_tokens(losses, dtype):
    """A workspace that holds 256 tokens at a time: the same losses and gradients of H, those of W within the order of the sum."""
    h, w, y, g = make(900, 777, 72, dtype)
    whole = losses.LossHead(900, 777, 72, DT[dtype])
    small = losses.LossHead(900, 777, 72, DT[dtype], max_workspace_bytes=1)
    assert small.workspace.numel() < whole.workspace.numel()
    a, b = whole.cross_entropy(h, w, y), small.cross_entropy(h, w, y)
    check(b, h, w, dtype, targets=y.cpu().numpy())
    assert (a.loss - b.loss).abs().max() <= 1e-5
    index, s = make_teacher(900, 777, 9, g)
    check(small.distill(h, w, index.to(torch.int32).cuda(), s.bfloat16().cuda(), temperature=1.5), h, w, dtype, tau=1.5,
          index=index.numpy(), teacher=s.bfloat16().double().numpy())


def test_offsets_beyond_32_bits(losses):
    """One piece whose probabilities take 5 GB: every loss, and the gradients' last rows, against fp64 on the device."""
    tokens, vocab, width = 20000, 131072, 64
    h, w, y, _ = make(tokens, vocab, width, "bf16")
    head = losses.LossHead(tokens, vocab, width, max_workspace_bytes=8 << 30)
    assert head.workspace.numel() > tokens * vocab * 2
    r = head.cross_entropy(h, w, y)
    w64, last, d_last = w.double(), vocab - 100, torch.zeros(100, width, dtype=torch.float64, device="cuda")
    for a in range(0, tokens, 2000):
        h64, at = h[a:a + 2000].double(), y[a:a + 2000, None]
        z = torch.mm(h64, w64.T.contiguous())
        lse = torch.logsumexp(z, 1)
        assert (r.loss[a:a + 2000] - (lse - z.gather(1, at)[:, 0])).abs().max() <= 1e-4
        dz = (z - lse[:, None]).exp().scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None])
        d_last += torch.mm(dz[:, last:].T.contiguous(), h64)
        d_hidden = torch.mm(dz, w64)
        assert (r.d_hidden[a:a + 2000].double() - d_hidden).norm() <= 5e-3 * d_hidden.norm()
    assert (r.d_weight[last:].double() - d_last).norm() <= 5e-3 * d_last.norm()


def test_one_gradient_at_a_time(losses):
    h, w, y, _ = make(100, 600, 64, "bf16")
    head = losses.LossHead(100, 600, 64)
    both = head.cross_entropy(h, w, y)
    only = head.cross_entropy(h, w, y, gradients=("hidden",))
    assert only.d_weight is None and torch.equal(only.d_hidden, both.d_hidden)
    only = head.cross_entropy(h, w, y, gradients=["weight"])
    assert only.d_hidden is None and torch.equal(only.d_weight, both.d_weight)


def test_no_tokens(losses):
    head = losses.LossHead(16, 100, 32)
    w = torch.randn(100, 32, device="cuda").bfloat16()
    r = head.cross_entropy(w.new_empty(0, 32), w, torch.empty(0, dtype=torch.int64, device="cuda"))
    assert r.loss.shape == (0,) and r.d_hidden.shape == (0, 32) and not r.d_weight.any()


def test_gradient_against_differences(losses):
    """fp32: the change of the loss along a direction is the gradient's product with it.  A step of 1e-2 in units of the direction's
    scale leaves a truncation error of about its square and the losses' rounding, 1e-6 over the step."""
    h, w, y, g = make(50, 400, 48, "f32")
    head = losses.LossHead(50, 400, 48, torch.float32)
    index, s = (t.cuda() for t in make_teacher(50, 400, 6, g))
    for call in (lambda a, b: head.cross_entropy(a, b, y), lambda a, b: head.distill(a, b, index, s, temperature=1.5)):
        r = call(h, w)
        for which, d in ((0, r.d_hidden), (1, r.d_weight)):
            way = torch.randn((h, w)[which].shape, generator=g).cuda()
            way = (way / 7 + d / d.norm() * way.norm() / 7) * (0.05 if which else 1.0)       # along the gradient as well
            step = 1e-2
            up, down = (call(*((h + e * way, w) if which == 0 else (h, w + e * way))).loss.double().sum() for e in (step, -step))
            assert abs((up - down) / (2 * step) - (d.double() * way.double()).sum()) <= 2e-3 * (d.double() * way.double()).abs().sum()


def test_repeats_are_bitwise_equal_and_streams_work(losses):
    h, w, y, _ = make(200, 3000, 128, "bf16")
    head = losses.LossHead(200, 3000, 128)
    a = head.cross_entropy(h, w, y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = head.cross_entropy(h, w, y)
    torch.cuda.current_stream().wait_stream(side)
    for x, z in zip(a, b):
        assert torch.equal(x, z)
    del head                                                # its memory is not handed out before the side stream is done with it


def test_replays_of_a_captured_call(losses):
    h, w, y, _ = make(100, 1000, 64, "bf16")
    head = losses.LossHead(100, 1000, 64)
    head.cross_entropy(h, w, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = head.cross_entropy(h, w, y)
    for k in range(3):
        h.mul_(1.0 - 0.25 * k)
        graph.replay()
        torch.cuda.synchronize()
        want = losses.LossHead(100, 1000, 64).cross_entropy(h, w, y)
        torch.cuda.synchronize()
        for a, b in zip(r, want):
            assert torch.equal(a, b)


def test_refusals(losses):
    from paper_2502_16982_amd.binding import MuonError
    h, w, y, _ = make(10, 50, 16, "bf16")
    head = losses.LossHead(10, 50, 16)
    s = torch.zeros(10, 3, device="cuda")
    i = torch.zeros(10, 3, dtype=torch.int64, device="cuda")
    for status, call in (
            (-2, lambda: head.cross_entropy(h.half(), w.half(), y)), (-2, lambda: head.cross_entropy(h, w.float(), y)),
            (-1, lambda: head.cross_entropy(h[:, :8], w, y)), (-1, lambda: head.cross_entropy(h, w, y[:5])),
            (-2, lambda: head.cross_entropy(h, w, y.to(torch.int16))), (-1, lambda: head.cross_entropy(h, w, y.cpu())),
            (-1, lambda: head.cross_entropy(h.T.contiguous().T, w, y)), (-1, lambda: head.cross_entropy(h[:1].expand(10, 16), w, y)),
            (-2, lambda: head.cross_entropy(h, w, y, token_scale=torch.ones(10, device="cuda").double())),
            (-1, lambda: head.cross_entropy(h, w, y, token_scale=torch.ones(11, device="cuda"))),
            (-1, lambda: head.distill(h, w, i[:, :2], s)), (-1, lambda: head.distill(h, w, i, s, temperature=0.0)),
            (-1, lambda: head.distill(h, w, i, s, temperature=float("nan"))), (-2, lambda: head.distill(h, w, i, s.half())),
            (-1, lambda: head.distill(h, w, i[:, :0], s[:, :0]))):
        with pytest.raises(MuonError) as e:
            call()
        assert e.value.status == status
    with pytest.raises(ValueError):
        head.cross_entropy(h, w, y, gradients=("logits",))

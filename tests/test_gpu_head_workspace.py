"""Workspaces of the head's losses on the device: smaller calls in a larger call's, and what outlives what."""
import pytest
import torch

from tests.head_pieces import PIECES

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(tokens, vocab, width, dtype="bf16", seed=0):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(vocab, width, generator=g) * 0.05
    h = torch.randn(tokens, width, generator=g)
    y = torch.randint(vocab, (tokens,), generator=g)
    return h.to(DT[dtype]).cuda(), w.to(DT[dtype]).cuda(), y.cuda()


def want64(h, w, y, scale=None):
    """loss, d_hidden, d_weight of the sum in fp64 on the device."""
    h64, w64, at = h.double(), w.double(), y[:, None]
    z = torch.mm(h64, w64.T.contiguous())
    lse = torch.logsumexp(z, 1)
    dz = (z - lse[:, None]).exp()
    dz.scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None])
    if scale is not None:
        dz *= scale.double()[:, None]
    return lse - z.gather(1, at)[:, 0], torch.mm(dz, w64), torch.mm(dz.T.contiguous(), h64)


@pytest.mark.parametrize("limit", [0, 27 << 20])
def test_fewer_tokens_in_the_workspace_of_more(limit):
    """1680 tokens take K in one run, 1260 would take it in several; what the larger call was given serves the smaller one, through the C
    ABI as well.  bf16: gradients as a whole within 5e-3, dz and the result rounded once each."""
    from paper_2502_16982_amd import binding
    tokens, fewer, vocab, width = 1680, 1260, 3817, 4096
    h, w, y = make(tokens, vocab, width)
    head = binding.muon_head(h.data_ptr(), w.data_ptr(), width, width, tokens, vocab, width, 1, 0)
    workspace = torch.empty(binding.muon_head_workspace_bytes(head, 1, 3, limit), dtype=torch.uint8, device="cuda")
    for n in (tokens, fewer, 1):
        loss = torch.empty(n, device="cuda")
        dh, dw = torch.empty_like(h[:n]), torch.empty_like(w)
        head = binding.muon_head(h.data_ptr(), w.data_ptr(), width, width, n, vocab, width, 1, 0)
        binding.muon_cross_entropy(head, y.data_ptr(), 8, 0, loss.data_ptr(), 0, dh.data_ptr(), dw.data_ptr(), workspace.data_ptr(),
                                   workspace.numel(), torch.cuda.current_stream().cuda_stream)
        want, want_h, want_w = want64(h[:n], w, y[:n])
        assert (loss - want).abs().max() <= 1e-4
        for got, ref in ((dh, want_h), (dw, want_w)):
            assert (got.double() - ref).norm() <= 5e-3 * ref.norm()


def test_results_do_not_depend_on_earlier_calls():
    """Pieces of tokens of one size, also where an earlier call of a larger vocabulary, whose smallest workspace is beyond the limit, left room
    for larger ones."""
    from paper_2502_16982_amd import losses
    h, w, y = make(9000, 600, 64, "f32")
    fresh = losses.LossHead(9000, 600, 64, torch.float32, max_workspace_bytes=30 << 20).cross_entropy(h, w, y)
    head = losses.LossHead(9000, 600, 64, torch.float32, max_workspace_bytes=30 << 20)
    head.cross_entropy(*make(9000, 20000, 64, "f32"))
    assert head.workspace.numel() > 60 << 20
    again = head.cross_entropy(h, w, y)
    for a, b in zip(fresh, again):
        assert torch.equal(a, b)


def test_replays_after_a_larger_call():
    """Calls that need more memory than a captured one replace the workspace, not the memory that the graph writes to."""
    from paper_2502_16982_amd import losses
    h, w, y = make(100, 1000, 64)
    head = losses.LossHead(100, 1000, 64)
    head.cross_entropy(h, w, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = head.cross_entropy(h, w, y)
    captured = head.workspace.data_ptr()
    index, s = torch.randint(1000, (100, 600), device="cuda"), torch.randn(100, 600, device="cuda")
    head.distill(h, w, index, s)
    assert head.workspace.data_ptr() != captured
    head.cross_entropy(*make(100, 40000, 64))
    others = [torch.full((n,), 3, dtype=torch.uint8, device="cuda") for n in (1 << 16, 1 << 18, 1 << 19, 1 << 20, 1 << 21)]
    want = losses.LossHead(100, 1000, 64).cross_entropy(h, w, y)
    for _ in range(3):
        for t in r[:2]:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(r, want):
            assert torch.equal(a, b)
    assert all((t == 3).all() for t in others)


def blocks(x):
    """Norms of the 64 x 64 blocks of a matrix."""
    rows, cols = -(-x.shape[0] // 64) * 64, -(-x.shape[1] // 64) * 64
    full = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
    full[:x.shape[0], :x.shape[1]] = x
    return full.view(rows // 64, 64, cols // 64, 64).square().sum((1, 3)).sqrt()


@pytest.mark.parametrize("name", PIECES)
@pytest.mark.parametrize("kind", ["cross entropy", "distillation"])
def test_pieces_with_scales(name, kind):
    """Several pieces of tokens whose scales differ, so that a piece that takes another's shows; block by block of 64 x 64 against fp64:
    twice the bar of a whole gradient in a block (fewer roundings average), never held to less than a thousandth of the typical block."""
    from paper_2502_16982_amd import losses
    tokens, vocab, width, f32, limit = PIECES[name]
    h, w, y = make(tokens, vocab, width, "f32" if f32 else "bf16")
    scale = (1.0 + torch.arange(tokens, device="cuda") / 500.0) / tokens
    y[::9] = -100
    head = losses.LossHead(tokens, vocab, width, h.dtype, max_workspace_bytes=limit, top=1)
    h64, w64, there = h.double(), w.double(), (y >= 0)[:, None]
    z = torch.mm(h64, w64.T.contiguous())
    if kind == "cross entropy":
        r = head.cross_entropy(h, w, y, token_scale=scale)
        tau, at, q = 1.0, y.clamp(min=0)[:, None], there.double()
    else:
        tau = 2.0
        at = torch.stack([y, (y + 7) % vocab], 1)
        s = torch.randn(tokens, 2, generator=torch.Generator().manual_seed(5)).cuda()
        r = head.distill(h, w, torch.where(there, at, -1), s, temperature=tau, token_scale=scale)
        at, q = at.clamp(min=0), torch.softmax(s.double() / tau, 1) * there
        z /= tau
    lse = torch.logsumexp(z, 1, keepdim=True)
    loss = tau * tau * (torch.special.xlogy(q, q) + q * (lse - z.gather(1, at))).sum(1)
    assert (r.loss - loss).abs().max() <= 1e-4
    dz = (z - lse).exp() * there
    dz.scatter_add_(1, at, -q)
    dz *= tau * scale.double()[:, None]
    bar = 2 * (1e-5 if f32 else 5e-3)
    for got, want in ((r.d_hidden, torch.mm(dz, w64)), (r.d_weight, torch.mm(dz.T.contiguous(), h64))):
        off, size = blocks(got.double() - want), blocks(want)
        assert (off <= bar * size.clamp(min=1e-3 * float(size.square().mean().sqrt()))).all()

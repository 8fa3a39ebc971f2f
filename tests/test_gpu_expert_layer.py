"""A mixture's layer for few tokens through the HIP library against the fp64 oracle on the same inputs.

Tolerances: a sum of n products in fp32 is off by less than (4 + sqrt n) 2^-23 of the sum of magnitudes (rounding errors of the sum
average); bf16 rounds h by at most 2^-8 of it (eps / 2) and out by 2^-8; what that adds up to in each element is the oracle's bound.
"""
import numpy as np
import pytest
import torch

from oracle import layer_oracle

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def experts():
    from paper_2502_16982_amd import experts as e
    return e


def as64(t):
    return None if t is None else t.detach().float().cpu().numpy().astype(np.float64)


def make(tokens, width, inner, n, top, dtype, gated=True, dropped=0.0, seed=0):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g) * std).to(DT[dtype]).cuda()

    expert = torch.stack([torch.randperm(n, generator=g)[:top] for _ in range(tokens)]) if top <= n else torch.randint(n, (tokens, top), generator=g)
    expert = torch.where(torch.rand(tokens, top, generator=g) < dropped, -1, expert).cuda()
    weights = torch.rand(tokens, top, generator=g).cuda()
    return (normal(tokens, width), normal(n, width, inner, std=width ** -0.5), normal(n, inner, width, std=inner ** -0.5), expert, weights,
            normal(n, width, inner, std=width ** -0.5) if gated else None)


def check(out, x, up, down, expert, weights, gate, activation="silu"):
    bf16 = x.dtype == torch.bfloat16
    want, bound = layer_oracle.layer(as64(x), as64(up), as64(down), expert.cpu().numpy(), as64(weights), as64(gate), activation, 2.0 ** -23,
                                     2.0 ** -8 if bf16 else 0.0)
    assert out.shape == x.shape and out.dtype == x.dtype
    got = as64(out)
    limit = bound + np.abs(want) * (2.0 ** -8 if bf16 else 2.0 ** -23) * 1.01 + 1e-37
    assert (np.abs(got - want) <= limit).all(), np.max(np.abs(got - want) / limit)


SIZES = [(1, 1, 1, 1, 1), (1, 8, 8, 2, 1), (3, 31, 7, 4, 2), (2, 33, 129, 3, 3), (1, 2048, 1408, 8, 6), (5, 777, 333, 16, 2), (17, 96, 130, 2, 1),
         (33, 160, 64, 2, 2), (40, 128, 128, 1, 1), (64, 257, 200, 12, 5), (7, 4, 3, 5, 2), (1, 300, 5000, 4, 4), (2, 5000, 40, 4, 1), (200, 64, 48, 8, 3)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_sizes(experts, sizes, gated, dtype):
    tokens, width, inner, n, top = sizes
    x, up, down, expert, weights, gate = make(tokens, width, inner, n, top, dtype, gated, dropped=0.2 if tokens > 2 else 0.0)
    check(experts.layer(x, up, down, expert, weights, gate=gate), x, up, down, expert, weights, gate)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forms(experts, dtype):
    """int32 experts, no weights, relu, an expert named twice, tokens without any, indexes beyond the experts."""
    x, up, down, expert, weights, gate = make(9, 72, 100, 6, 3, dtype)
    for act in ("silu", "relu"):
        for g in (gate, None):
            check(experts.layer(x, up, down, expert.to(torch.int32), None, gate=g, activation=act), x, up, down, expert, None, g, act)
    expert[0, :] = 2
    expert[1, :] = -1
    expert[2, 0], expert[3, 1] = 6, 1 << 40
    out = experts.layer(x, up, down, expert, weights, gate=gate)
    check(out, x, up, down, expert, weights, gate)
    assert (out[1] == 0).all()
    assert (experts.layer(x, up, down, torch.full_like(expert, -5), weights) == 0).all()
    assert experts.layer(x[:0], up, down, expert[:0], weights[:0]).shape == (0, 72)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_alignment(experts, dtype):
    """Rows apart, experts apart, at any alignment of an element; halves of one matrix as gate and up."""
    dt = DT[dtype]
    x, up, down, expert, weights, gate = make(6, 75, 50, 4, 2, dtype)
    both = torch.zeros(4, 75, 103, dtype=dt, device="cuda")
    both[:, :, 1:51], both[:, :, 52:102] = gate, up
    wide = torch.zeros(4, 53, 80, dtype=dt, device="cuda")
    wide[:, 2:52, 3:78] = down
    rows = torch.zeros(6, 200, dtype=dt, device="cuda")
    rows[:, 5:80] = x
    a = experts.layer(rows[:, 5:80], both[:, :, 52:102], wide[:, 2:52, 3:78], expert, weights, gate=both[:, :, 1:51])
    b = experts.layer(x, up, down, expert, weights, gate=gate)
    assert torch.equal(a, b)
    check(b, x, up, down, expert, weights, gate)
    one = experts.layer(x, up[:1].expand(4, -1, -1), down[:1].expand(4, -1, -1), expert, weights)
    check(one, x, up[:1].expand(4, -1, -1), down[:1].expand(4, -1, -1), expert, weights, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite_stay_where_they_are(experts, dtype):
    """A token's reach its own row only, an expert's its own tokens; what no token goes to is not read into anything."""
    x, up, down, expert, weights, gate = make(20, 70, 90, 5, 2, dtype)
    expert[:] = torch.tensor([0, 1], device="cuda")
    expert[7] = torch.tensor([2, 1], device="cuda")
    want = experts.layer(x, up, down, expert, weights, gate=gate)
    x2, up2, down2 = x.clone(), up.clone(), down.clone()
    x2[3, 69] = float("nan")
    up2[2, 69, 89], down2[2] = float("inf"), float("nan")
    up2[3:], down2[3:] = float("nan"), float("inf")
    got = experts.layer(x2, up2, down2, expert, weights, gate=gate)
    assert got[3].isnan().all() and got[7].isnan().all()
    rest = [t for t in range(20) if t not in (3, 7)]
    assert torch.equal(got[rest], want[rest])


def test_weights_of_dropped_pairs_do_not_count(experts):
    x, up, down, expert, weights, gate = make(4, 64, 64, 4, 2, "bf16")
    expert[:, 1] = -1
    want = experts.layer(x, up, down, expert, weights, gate=gate)
    weights[:, 1] = float("nan")
    assert torch.equal(experts.layer(x, up, down, expert, weights, gate=gate), want)


def test_as_sorted_rows_go(experts):
    """The way over sort, dispatch, products and combine, on the same tokens."""
    x, up, down, expert, weights, gate = make(24, 256, 128, 8, 2, "f32")
    routing = experts.sort_by_expert(expert, 8)
    rows = experts.dispatch(x, routing)
    y = torch.zeros_like(rows)
    edges = routing.offsets.tolist()
    for e in range(8):
        r = rows[edges[e]:edges[e + 1]]
        z = r @ gate[e]
        y[edges[e]:edges[e + 1]] = (z / (1 + (-z).exp()) * (r @ up[e])) @ down[e]
    a, b = experts.combine(y, weights, routing), experts.layer(x, up, down, expert, weights, gate=gate)
    assert (a - b).norm() <= 1e-5 * a.norm()


def test_matrices_beyond_32_bits(experts):
    """The last expert's matrices start beyond 2^32 elements."""
    n, width, inner = 1050, 2048, 2048
    up = torch.zeros(n, width, inner, dtype=torch.bfloat16, device="cuda")
    down = torch.zeros(n, inner, width, dtype=torch.bfloat16, device="cuda")
    x, u, d, _, weights, _ = make(2, width, inner, 1, 1, "bf16", gated=False)
    up[-1], down[-1] = u[0], d[0]
    expert = torch.tensor([[n - 1], [0]], device="cuda")
    out = experts.layer(x, up, down, expert, weights)
    check(out[:1], x[:1], u, d, torch.zeros(1, 1, dtype=torch.int64), weights[:1], None)
    assert (out[1] == 0).all()


def test_streams_and_capture(experts):
    x, up, down, expert, weights, gate = make(6, 512, 384, 16, 2, "bf16")
    want = experts.layer(x, up, down, expert, weights, gate=gate)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = experts.layer(x, up, down, expert, weights, gate=gate)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(there, want)
    held = x.clone(), expert.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = experts.layer(held[0], up, down, held[1], weights, gate=gate)
    for seed in range(3):
        x2, _, _, expert2, _, _ = make(6, 512, 384, 16, 2, "bf16", dropped=0.3, seed=10 + seed)
        held[0].copy_(x2)
        held[1].copy_(expert2)
        eager = experts.layer(x2, up, down, expert2, weights, gate=gate)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_autograd_is_warned_of(experts):
    x, up, down, expert, weights, gate = make(2, 16, 16, 2, 1, "f32")
    with pytest.warns(UserWarning, match="not recorded by autograd"):
        experts.layer(x.requires_grad_(), up, down, expert, weights)


def test_refusals(experts):
    from paper_2502_16982_amd.binding import MuonError
    x, up, down, expert, weights, gate = make(3, 16, 24, 4, 2, "f32")
    bad = [dict(x=x[:2]), dict(up=up[:, :15]), dict(down=down[:3]), dict(gate=gate.bfloat16()), dict(up=up.transpose(1, 2).contiguous().transpose(1, 2)),
           dict(weights=weights[:2]), dict(weights=weights.double()), dict(expert=expert.cpu()), dict(x=x.double(), up=up.double(), down=down.double(), gate=None),
           dict(up=up[0])]
    for over in bad:
        a = dict(x=x, up=up, down=down, expert=expert, weights=weights, gate=gate)
        a.update(over)
        with pytest.raises(MuonError):
            experts.layer(**a)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("activation", ["silu", "relu"])
@pytest.mark.parametrize("tokens,width,inner,n,top", [(4, 70, 90, 5, 2), (2, 700, 300, 4, 2), (1, 4096, 1408, 8, 8)])
def test_activations_of_nan_are_nan(experts, tokens, width, inner, n, top, activation, dtype):
    """NaN in a hidden state, and in one element of an expert's Gate or Up, reaches every element of the rows it is part of, wherever the activation is
    made: beside the first product, in the second one's operand or by a launch of its own."""
    x, up, down, expert, weights, gate = make(tokens, width, inner, n, top, dtype)
    expert[0] = torch.arange(top)
    nan = float("nan")
    for g in (gate, None):
        want = experts.layer(x, up, down, expert, weights, gate=g, activation=activation)
        check(want, x, up, down, expert, weights, g, activation)
        bad_x = x.clone()
        bad_x[0, width - 1] = nan
        got = experts.layer(bad_x, up, down, expert, weights, gate=g, activation=activation)
        assert got[0].isnan().all() and torch.equal(got[1:], want[1:])
        reached = (expert == 0).any(1)
        for which in ("up", "gate"):
            m = {"up": up, "gate": g}[which]
            if m is None:
                continue
            m = m.clone()
            m[0, 0, inner - 1] = nan
            got = experts.layer(x, m if which == "up" else up, down, expert, weights, gate=m if which == "gate" else g, activation=activation)
            assert got[reached].isnan().all() and torch.equal(got[~reached], want[~reached]), which


def silu64(z):
    return z / (1 + (-z).exp())


def test_most_blocks_of_the_products(experts):
    """As many experts, as many columns as there may be, both matrices by one block: 2^32 threads.  Experts share matrices of one row; bounds as the oracle's."""
    n, inner, g = 4096, 1 << 17, torch.Generator().manual_seed(8)
    up, gate, down = (torch.randn(inner, generator=g).cuda() for _ in range(3))
    x = torch.randn(n, 1, generator=g).cuda()
    weights = torch.rand(n, 1, generator=g).cuda()
    expert = torch.randperm(n, generator=g)[:, None].cuda()
    out = experts.layer(x, up.view(1, 1, inner).expand(n, 1, inner), down.view(1, inner, 1).expand(n, inner, 1), expert, weights,
                        gate=gate.view(1, 1, inner).expand(n, 1, inner))
    step = 2.0 ** -23
    for at in range(0, n, 256):
        x64, w64 = x[at:at + 256].double(), weights[at:at + 256, 0].double()
        u, z = x64 * up.double(), x64 * gate.double()
        lead = silu64(z)
        h = lead * u
        h_err = 1.1 * 5 * step * z.abs() * u.abs() * (1 + 5 * step) + lead.abs() * 5 * step * u.abs() + h.abs() * 2.0 ** -21
        y = h @ down.double()
        bound = w64 * (h_err @ down.double().abs() + (4 + inner ** 0.5) * step * (h.abs() @ down.double().abs()) + 2.0 ** -20 * y.abs()) + step * (w64 * y).abs()
        assert ((out[at:at + 256, 0].double() - w64 * y).abs() <= bound).all()


def test_most_blocks_of_the_join(experts):
    """As many tokens as there may be, of the largest width: 2^32 threads."""
    tokens, width, g = 1 << 14, 1 << 17, torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(tokens, width, generator=g, device="cuda", dtype=torch.bfloat16)
    up = (torch.randn(width, generator=g, device="cuda") * width ** -0.5).bfloat16()
    down = torch.randn(width, generator=g, device="cuda").bfloat16()
    out = experts.layer(x, up.view(1, width, 1), down.view(1, 1, width), torch.zeros(tokens, 1, dtype=torch.int32, device="cuda"))
    step = 2.0 ** -23
    for at in range(0, tokens, 1024):
        x64 = x[at:at + 1024].double()
        u = x64 @ up.double()
        h = silu64(u)
        h_err = 1.1 * (4 + width ** 0.5) * step * (x64.abs() @ up.double().abs()) + h.abs() * (2.0 ** -8 + 2.0 ** -21)
        scale = h_err + h.abs() * (5 * step + 2.0 ** -20 + 2.0 ** -8 * 1.01)             # bound of row t: scale_t |down|
        err = (out[at:at + 1024].double() - h[:, None] * down.double()).abs_()
        assert (err <= scale[:, None] * down.double().abs() + 1e-37).all()

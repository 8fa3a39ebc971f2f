"""The norm of gradients, clipping in place, and the scaled steps, against fp64 on the same inputs.

Tolerances.  Squares of fp32 (24 bits) and bf16 (8 bits) values are exact in a double's 53 bits; n of them summed in any order are off by at
most n 2^-53 relative, in runs far less: 1e-12 for the norm.  A scaled gradient: scale is rounded to fp32 (2^-24), the product to fp32
(2^-24, what bf16 rounds again by 2^-8): 2^-22.9 and 2^-7.99 relative of each element, below the normal range half a step of the type.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def clipping():
    from paper_2502_16982_amd import clipping as c
    return c


def make(sizes, dtypes, seed=0, std=1e-2):
    """Slices of one buffer per type, one behind the other, so that they start at any element."""
    gen = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        dt = dtypes[i % len(dtypes)]
        out.append((torch.randn(n, generator=gen) * std).to(dt))
    flats = {dt: torch.cat([g for g in out if g.dtype == dt] or [torch.zeros(0, dtype=dt)]).cuda() for dt in (BF16, F32)}
    at, grads = {BF16: 0, F32: 0}, []
    for g in out:
        grads.append(flats[g.dtype][at[g.dtype]:at[g.dtype] + g.numel()])
        at[g.dtype] += g.numel()
    return grads


def norm64(grads):
    return math.sqrt(sum(float(g.cpu().double().square().sum()) for g in grads))


def check_scaled(after, before, scale):
    for a, b in zip(after, before):
        want = b.cpu().double() * scale
        rel, least = (2.0 ** -7.99, 2.0 ** -134) if b.dtype == BF16 else (2.0 ** -22.9, 2.0 ** -150)
        assert (a.cpu().double() - want).abs().le(want.abs() * rel + least).all()


SIZES = [[1], [7], [0, 3, 0], [16384], [16383, 16385, 1], [65536 + 5], [1000003], list(range(1, 260)), [3] * 1000, [0], [100, 2000, 30000, 400000]]


@pytest.mark.parametrize("dtypes", [(BF16,), (F32,), (BF16, F32)])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_norm_and_clip(clipping, sizes, dtypes):
    grads = make(sizes, dtypes)
    before, want = [g.clone() for g in grads], norm64(grads)
    c = clipping.GradClipper(grads)
    r = c.scale(0.5 * want)
    assert r.norm.dtype == torch.float64 and r.scale.dtype == F32 and r.norm.shape == r.scale.shape == ()
    assert abs(float(r.norm) - want) <= 1e-12 * want
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    expect = 0.5 if want > 0 else 1.0
    assert abs(float(r.scale) - expect) <= 2.0 ** -24
    again = c.clip_(0.5 * want)
    assert float(again.norm) == float(r.norm) and float(again.scale) == float(r.scale)
    check_scaled(grads, before, expect)


def test_nothing_is_touched_below_the_limit(clipping):
    grads = make([5, 40000], (BF16, F32))
    before = [g.clone() for g in grads]
    c = clipping.GradClipper(grads)
    want = norm64(grads)
    for limit in (want * 1.0001, 1e30, math.inf):
        assert float(c.clip_(limit).scale) == 1.0
    assert float(c.scale().scale) == 1.0
    assert all(torch.equal(a, b) for a, b in zip(grads, before))


def test_limit_of_zero(clipping):
    grads = make([5, 40000], (BF16, F32))
    r = clipping.GradClipper(grads).clip_(0.0)
    assert float(r.scale) == 0.0 and all((g == 0).all() for g in grads)


@pytest.mark.parametrize("std", [1e30, 1e-30, 1e-42])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_squares_beyond_fp32(clipping, std, dtype):
    grads = make([100, 50001], (dtype,), std=std)
    want = norm64(grads)
    r = clipping.GradClipper(grads).clip_(want / 3)
    assert abs(float(r.norm) - want) <= 1e-12 * want


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_norms_that_are_not_finite_leave_the_gradients(clipping, bad):
    grads = make([5, 40000, 17], (BF16, F32))
    grads[1][39999] = bad
    before = [g.clone() for g in grads]
    r = clipping.GradClipper(grads).clip_(1.0)
    assert not math.isfinite(float(r.norm)) and float(r.scale) == 1.0
    assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(grads, before))


def test_many_partial_sums(clipping):
    """More than one launch holds in the last sum: they are joined in groups first."""
    g = torch.empty((32768 + 3) * 16384 + 11, dtype=BF16, device="cuda").normal_(0, 1e-2)
    want = math.sqrt(sum(float(p.double().square().sum()) for p in g.split(1 << 24)))
    r = clipping.GradClipper([g]).scale(1.0)
    assert abs(float(r.norm) - want) <= 1e-12 * want


def test_offsets_beyond_32_bits(clipping):
    n = (1 << 32) + 12345
    g = torch.zeros(n, dtype=BF16, device="cuda")
    g[:1], g[-1:], g[1 << 31] = 3.0, 4.0, 12.0
    c = clipping.GradClipper([g])
    r = c.clip_(6.5)
    assert float(r.norm) == 13.0 and float(r.scale) == 0.5
    assert float(g[0]) == 1.5 and float(g[-1]) == 2.0 and float(g[1 << 31]) == 6.0


def test_results_repeat_and_streams(clipping):
    grads = make([3001, 100003, 77], (BF16, F32))
    c = clipping.GradClipper(grads)
    first = c.scale(1e-3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = c.scale(1e-3)
    third = c.scale(1e-3)
    torch.cuda.synchronize()
    assert float(first.norm) == float(second.norm) == float(third.norm) and float(first.scale) == float(second.scale)


def test_captured(clipping):
    """Replays clip what is there, with eager calls of the same clipper between them."""
    grads = make([3001, 100003, 77], (BF16, F32))
    raw = [g.clone() for g in grads]
    c = clipping.GradClipper(grads)
    c.clip_(1.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = c.clip_(0.25)
    for k in range(4):
        for g, x in zip(grads, raw):
            g.copy_(x * (k + 1))
        want = [(x * (k + 1)) for x in raw]
        total = norm64(want)
        graph.replay()
        torch.cuda.synchronize()
        assert abs(float(r.norm) - total) <= 1e-12 * total
        check_scaled(grads, want, 0.25 / total)
        c.scale(1.0)


def test_scale_of_ones_own(clipping):
    grads = make([3001, 77], (BF16, F32))
    before = [g.clone() for g in grads]
    clipping.GradClipper(grads).scale_(torch.tensor([0.3], device="cuda"))
    check_scaled(grads, before, float(torch.tensor(0.3)))


@pytest.mark.parametrize("g_dtype", [BF16, F32])
@pytest.mark.parametrize("p_dtype", [BF16, F32])
def test_adamw_takes_the_scale(clipping, p_dtype, g_dtype):
    """Bit for bit the step on gradients scaled in fp32."""
    from paper_2502_16982_amd import binding
    gen = torch.Generator().manual_seed(3)
    sizes = [1, 5, 1023, 1024, 40001]
    quads = [[(torch.randn(n, generator=gen)).to(dt).cuda() for dt in (p_dtype, g_dtype, F32)] + [torch.rand(n, generator=gen).cuda()] for n in sizes]
    r = clipping.GradClipper([q[1] for q in quads]).scale(0.7)
    want = [[q[0].clone(), r.scale * q[1].float(), q[2].clone(), q[3].clone()] for q in quads]
    args = dict(lr=0.01, weight_decay=0.1, step=3, stream_ptr=torch.cuda.current_stream().cuda_stream)
    binding.muon_adamw_step([tuple(q) for q in want], **args)
    binding.muon_adamw_step([tuple(q) for q in quads], grad_scale=r.scale, **args)
    for a, b in zip(quads, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2]) and torch.equal(a[3], b[3])


@pytest.mark.parametrize("ns", ["f32", "bf16"])
@pytest.mark.parametrize("g_dtype", [BF16, F32])
def test_muon_takes_the_scale(clipping, ns, g_dtype):
    """Bit for bit the step on gradients scaled in fp32."""
    from paper_2502_16982_amd import binding
    gen = torch.Generator().manual_seed(4)
    shapes = [(64, 96), (200, 70), (128, 128)]
    mats = [[torch.randn(s, generator=gen).cuda(), torch.randn(s, generator=gen).to(g_dtype).cuda(), torch.randn(s, generator=gen).cuda()] for s in shapes]
    r = clipping.GradClipper([m[1] for m in mats]).scale(2.0)
    want = [[m[0].clone(), r.scale * m[1].float(), m[2].clone()] for m in mats]
    hp = binding.default_hparams(lr=0.02, weight_decay=0.1)
    a, b = binding.MuonStepper(mats, ns_dtype=ns), binding.MuonStepper(want, ns_dtype=ns)
    a.step(hp, grad_scale=r.scale)
    b.step(hp)
    for x, y in zip(mats, want):
        assert torch.equal(x[0], y[0]) and torch.equal(x[2], y[2])

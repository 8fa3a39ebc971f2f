"""The experts' sort, dispatch and combine through the HIP library against plain loops in fp64.

Tolerances: the sort and what only moves rows are exact.  A sum of `top` products in fp32 is off by at most (top + 1) 2^-24 of the sum
of magnitudes, and its rounding by 2^-24 (fp32) or 2^-8 (bf16, whose significand has 8 bits) of the result; a dot product of D terms by (4 + sqrt(D)) 2^-23 of the
sum of magnitudes (rounding errors average)."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as ex

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ROUND = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def experts():
    from paper_2502_16982_amd import experts as e
    return e


def as64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def fast_sort(expert, n):
    """What ex.sort_pairs says, for many pairs."""
    flat = expert.reshape(-1)
    keep = np.flatnonzero((flat >= 0) & (flat < n))
    order = keep[np.argsort(flat[keep], kind="stable")]
    position, source = -np.ones(flat.size, np.int64), -np.ones(flat.size, np.int64)
    position[order], source[:order.size] = np.arange(order.size), order
    return position.reshape(expert.shape), source, np.concatenate([[0], np.cumsum(np.bincount(flat[keep], minlength=n))])


def random_experts(tokens, top, n, seed, dropped=0.2):
    g = np.random.default_rng(seed)
    e = np.minimum(g.integers(0, n, (tokens, top)), g.integers(0, n, (tokens, top)))        # the first ones are liked more
    return np.where(g.random((tokens, top)) < dropped, g.choice([-1, -7, n, n + 5], (tokens, top)), e)


@pytest.mark.parametrize("tokens,top,n", [(1, 1, 1), (1, 6, 64), (7, 3, 5), (64, 2, 2), (341, 6, 66), (2048, 1, 8), (683, 3, 130), (3000, 8, 64),
                                          (70000, 8, 128), (5000, 64, 1000), (257, 9, 4096)])
@pytest.mark.parametrize("wide", [False, True])
def test_sort(experts, tokens, top, n, wide):
    e = random_experts(tokens, top, n, tokens)
    r = experts.sort_by_expert(torch.tensor(e, dtype=torch.int64 if wide else torch.int32, device="cuda"), n)
    want = ex.sort_pairs(e, n) if e.size * n < 20000 else fast_sort(e, n)
    for got, ref in zip(r, want):
        assert got.dtype == torch.int32 and np.array_equal(got.cpu().numpy(), ref)


def test_sort_of_one_expert_and_of_none(experts):
    one = torch.full((3000, 2), 3, dtype=torch.int32, device="cuda")
    r = experts.sort_by_expert(one, 5)
    assert torch.equal(r.source, torch.arange(6000, dtype=torch.int32, device="cuda")) and r.offsets.tolist() == [0, 0, 0, 0, 6000, 6000]
    r = experts.sort_by_expert(torch.full_like(one, -1), 5)
    assert (r.position == -1).all() and (r.source == -1).all() and not r.offsets.any()
    r = experts.sort_by_expert(one[:0], 5)
    assert r.position.shape == (0, 2) and not r.offsets.any()


def test_large_wide_indices_are_dropped(experts):
    """64-bit experts whose low 32 bits would be valid ones."""
    e = torch.tensor([[1 << 32, 1], [(1 << 33) + 1, 0]], dtype=torch.int64, device="cuda")
    assert experts.sort_by_expert(e, 2).position.tolist() == [[-1, 1], [-1, 0]]


CASES = [(1, 1, 1, 1), (1, 6, 64, 256), (5, 2, 3, 7), (33, 3, 8, 24), (64, 6, 64, 1409), (130, 8, 16, 512), (200, 4, 8, 2048), (77, 64, 70, 66), (50, 5, 4, 5000)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,top,n,width", CASES)
@pytest.mark.parametrize("dropped", [0.0, 0.3, 1.0])
def test_rows(experts, tokens, top, n, width, dtype, dropped):
    e = random_experts(tokens, top, n, 3, dropped)
    position, _, offsets = fast_sort(e, n)
    r = experts.sort_by_expert(torch.tensor(e, dtype=torch.int32, device="cuda"), n)
    g = torch.Generator().manual_seed(width)
    x, d_out = (torch.randn(tokens, width, generator=g).to(DT[dtype]).cuda() for _ in range(2))
    rows = torch.randn(tokens * top, width, generator=g).to(DT[dtype]).cuda()
    rows[int(offsets[-1]):] = float("nan")                  # behind the last pair's row: never read
    w = torch.rand(tokens, top, generator=g).cuda() - 0.3
    got = experts.dispatch(x, r)
    assert np.array_equal(as64(got), ex.dispatch(as64(x), position))
    rows64, w64 = np.nan_to_num(as64(rows)), as64(w)
    for weights, out in ((w64, experts.combine(rows, w, r)), (None, experts.dispatch_backward(rows, r))):
        want = ex.combine(rows64, weights, position)
        size = ex.combine(np.abs(rows64), None if weights is None else np.abs(weights), position)
        assert (np.abs(as64(out) - want) <= (top + 1) * 2.0 ** -24 * size + ROUND[dtype] * np.abs(want) * (1 + 2.0 ** -8)).all()
    d_rows, d_w = experts.combine_backward(d_out, rows, w, r)
    want_rows, want_w = ex.combine_backward(as64(d_out), rows64, w64, position)
    _, size = ex.combine_backward(np.abs(as64(d_out)), np.abs(rows64), w64, position)
    assert (np.abs(as64(d_rows) - want_rows) <= (2.0 ** -24 + ROUND[dtype]) * np.abs(want_rows)).all()
    assert (np.abs(as64(d_w) - want_w) <= (4 + np.sqrt(width)) * 2.0 ** -23 * size).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("extra,start", [(8, 0), (8, 4), (3, 1)])
def test_strides_and_alignment(experts, dtype, extra, start):
    e = random_experts(40, 3, 8, 5)
    r = experts.sort_by_expert(torch.tensor(e, dtype=torch.int32, device="cuda"), 8)
    g = torch.Generator().manual_seed(1)
    wide = torch.randn(40, 264 + extra, generator=g).to(DT[dtype]).cuda()
    x = wide[:, start:start + 264]
    rows, w = experts.dispatch(x.contiguous(), r), torch.rand(40, 3, generator=g).cuda()
    assert torch.equal(experts.dispatch(x, r), rows)
    for a, b in zip(experts.combine_backward(x, rows, w, r), experts.combine_backward(x.contiguous(), rows, w, r)):
        assert torch.allclose(a, b, rtol=2.0 ** -20, atol=1e-4)         # another width of access sums in another order


def test_offsets_beyond_32_bits(experts):
    """Rows of 6.9 GB: their last ones go where they belong, both ways."""
    tokens, top, width = 70000, 6, 8192
    e = random_experts(tokens, top, 64, 9, 0.0)
    position, source, _ = fast_sort(e, 64)
    r = experts.sort_by_expert(torch.tensor(e, dtype=torch.int32, device="cuda"), 64)
    x = torch.randn(tokens, width, device="cuda").bfloat16()
    rows = experts.dispatch(x, r)
    some = torch.tensor(np.concatenate([np.arange(0, tokens * top, 9973), np.arange(tokens * top - 50, tokens * top)]), device="cuda")
    assert torch.equal(rows[some], x[torch.tensor(source, device="cuda")[some] // top])
    back = experts.dispatch_backward(rows, r)
    assert torch.equal(back, (6 * x.float()).bfloat16())                    # six copies of the token's own row
    w = torch.rand(tokens, top, device="cuda")
    d_rows, d_w = experts.combine_backward(x, rows, w, r)
    want = x.double().square().sum(1, keepdim=True)
    assert ((d_w - want).abs() <= (4 + width ** 0.5) * 2.0 ** -23 * want).all()
    at = torch.tensor(position[-1], device="cuda")
    assert torch.equal(d_rows[at], (w[-1, :, None] * x[-1].float()).bfloat16())


def test_gradients_against_differences(experts):
    """combine is linear in rows and in weights: one difference is exact but for rounding."""
    e = random_experts(60, 4, 9, 2)
    r = experts.sort_by_expert(torch.tensor(e, dtype=torch.int32, device="cuda"), 9)
    g = torch.Generator().manual_seed(2)
    rows, step = (torch.randn(240, 32, generator=g).cuda() for _ in range(2))
    w, w_step = (torch.rand(60, 4, generator=g).cuda() for _ in range(2))
    d_out = torch.randn(60, 32, generator=g).cuda()
    rows[r.offsets[-1]:] = 0
    d_rows, d_w = experts.combine_backward(d_out, rows, w, r)
    loss = lambda a, b: (experts.combine(a, b, r).double() * d_out).sum()  # noqa: E731
    assert abs(loss(rows + step, w) - loss(rows, w) - (d_rows.double() * step).sum()) <= 1e-3
    assert abs(loss(rows, w + w_step) - loss(rows, w) - (d_w.double() * w_step).sum()) <= 1e-3
    x = torch.randn(60, 32, generator=g).cuda()
    assert abs((experts.dispatch(x, r).double() * rows).sum() - (experts.dispatch_backward(rows, r).double() * x).sum()) <= 1e-3


def test_positions_outside_the_rows_count_as_dropped(experts):
    r = experts.sort_by_expert(torch.zeros(4, 2, dtype=torch.int32, device="cuda"), 1)
    r.position[1, 1], r.position[2, 0] = 8, 2 ** 31 - 1
    x = torch.ones(4, 16, device="cuda")
    experts.dispatch(x, r)
    assert experts.dispatch_backward(torch.ones(8, 16, device="cuda"), r)[:, 0].tolist() == [2.0, 1.0, 1.0, 2.0]


def test_replays_of_captured_calls(experts):
    e = torch.tensor(random_experts(900, 6, 64, 4), dtype=torch.int32, device="cuda")
    x = torch.randn(900, 64, device="cuda")
    experts.dispatch(x, experts.sort_by_expert(e, 64))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = experts.sort_by_expert(e, 64)
        rows = experts.dispatch(x, r)
    for k in range(3):
        e.copy_(torch.tensor(random_experts(900, 6, 64, 10 + k), dtype=torch.int32))
        x.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        want = experts.sort_by_expert(e, 64)
        for a, b in zip(r, want):
            assert torch.equal(a, b)
        assert torch.equal(rows, experts.dispatch(x, want))


def test_refusals(experts):
    from paper_2502_16982_amd.binding import MuonError
    e = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    r = experts.sort_by_expert(e, 3)
    x, w = torch.zeros(4, 16, device="cuda"), torch.zeros(4, 2, device="cuda")
    rows = torch.zeros(8, 16, device="cuda")
    for status, call in (
            (-2, lambda: experts.sort_by_expert(e.float(), 3)), (-1, lambda: experts.sort_by_expert(e, 0)),
            (-1, lambda: experts.sort_by_expert(e, 4097)), (-1, lambda: experts.sort_by_expert(e.T, 3)),
            (-1, lambda: experts.sort_by_expert(e.cpu(), 3)), (-1, lambda: experts.sort_by_expert(e.new_zeros(2, 65), 3)),
            (-1, lambda: experts.dispatch(x[:3], r)), (-2, lambda: experts.dispatch(x.half(), r)),
            (-1, lambda: experts.dispatch(x.T.contiguous().T, r)), (-1, lambda: experts.combine(rows[:7], w, r)),
            (-2, lambda: experts.combine(rows, w.bfloat16(), r)), (-1, lambda: experts.combine(rows, w[:, :1], r)),
            (-1, lambda: experts.combine_backward(x[:, :8], rows, w, r)), (-2, lambda: experts.combine_backward(x.bfloat16(), rows, w, r)),
            (-2, lambda: experts.dispatch(x, experts.Routing(r.position.long(), r.source, r.offsets)))):
        with pytest.raises(MuonError) as err:
            call()
        assert err.value.status == status

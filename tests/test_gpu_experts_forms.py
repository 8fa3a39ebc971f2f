"""The experts' kernels where a launch goes on to further tokens, and rows of any alignment bit for bit."""
import warnings

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def experts():
    from paper_2502_16982_amd import experts as e
    return e


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_tokens_than_a_launch_has_at_a_time(experts, dtype):
    """2^24 + 5 tokens of one choice: the last ones go through a block that had others before.  Rows of one element: all of it exact but for
    the rounding of a product."""
    tokens = (1 << 24) + 5
    g = torch.Generator(device="cuda").manual_seed(1)
    e = torch.randint(-1, 3, (tokens, 1), generator=g, device="cuda", dtype=torch.int32)
    r = experts.sort_by_expert(e, 3)
    key = torch.where(e[:, 0] >= 0, e[:, 0], 3)
    order = torch.sort(key, stable=True).indices
    count = int((e >= 0).sum())
    assert r.offsets.tolist() == [0, *((key[:, None] == torch.arange(3, device="cuda")).sum(0).cumsum(0).tolist())]
    assert torch.equal(r.source[:count].long(), order[:count]) and (r.source[count:] == -1).all()
    assert torch.equal(r.position[order[:count], 0].long(), torch.arange(count, device="cuda")) and (r.position[order[count:]] == -1).all()
    x, d_out = (torch.randn(tokens, 1, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    rows = experts.dispatch(x, r)
    assert torch.equal(rows[:count], x[order[:count]]) and not rows[count:].any()
    w = torch.rand(tokens, 1, generator=g, device="cuda")
    there = e >= 0
    assert torch.equal(experts.combine(rows, w, r), torch.where(there, w * x.float(), 0.0).to(DT[dtype]))
    assert torch.equal(experts.dispatch_backward(rows, r), torch.where(there, x.float(), 0.0).to(DT[dtype]))
    d_rows, d_w = experts.combine_backward(d_out, rows, w, r)
    assert torch.equal(d_w, torch.where(there, d_out.float() * x.float(), 0.0))
    assert torch.equal(d_rows[:count], (w * d_out.float()).to(DT[dtype])[order[:count]]) and not d_rows[count:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [1, 66, 264, 1409])
@pytest.mark.parametrize("extra,start", [(8, 0), (8, 4), (3, 1)])
def test_alignment_changes_no_bit(experts, dtype, width, extra, start):
    """Rows move in pieces of 16 bytes at any alignment: sums run in the same order whatever the stride."""
    g = torch.Generator().manual_seed(1)
    e = torch.randint(-1, 8, (40, 3), generator=g).to(torch.int32).cuda()
    r = experts.sort_by_expert(e, 8)
    x = torch.randn(40, width + extra, generator=g).to(DT[dtype]).cuda()[:, start:start + width]
    rows, w = torch.randn(120, width, generator=g).to(DT[dtype]).cuda(), torch.rand(40, 3, generator=g).cuda()
    assert torch.equal(experts.dispatch(x, r), experts.dispatch(x.contiguous(), r))
    for a, b in zip(experts.combine_backward(x, rows, w, r), experts.combine_backward(x.contiguous(), rows, w, r)):
        assert torch.equal(a, b)
    # ... and rows and results at an address that is no multiple of 16 bytes
    odd = torch.empty(120 * width + 1, dtype=DT[dtype], device="cuda")[1:].view(120, width)
    odd.copy_(rows)
    assert torch.equal(experts.combine(odd, w, r), experts.combine(rows, w, r))
    for a, b in zip(experts.combine_backward(x, odd, w, r), experts.combine_backward(x, rows, w, r)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("pairs", [1, 63, 64, 65, 255, 256, 257, 511, 513, 1023, 1024, 1025, 2047, 2049, 131071, 131073])
@pytest.mark.parametrize("n", [1, 66, 4096])
def test_sort_at_the_ends_of_its_blocks(experts, pairs, n):
    g = torch.Generator(device="cuda").manual_seed(pairs)
    e = torch.randint(-1, n + 1, (pairs, 1), generator=g, device="cuda", dtype=torch.int32)
    r = experts.sort_by_expert(e, n)
    key = torch.where((e[:, 0] >= 0) & (e[:, 0] < n), e[:, 0], n).long()
    order = torch.sort(key, stable=True).indices
    count = int((key < n).sum())
    assert torch.equal(r.source[:count].long(), order[:count]) and (r.source[count:] == -1).all()
    assert torch.equal(r.position[order[:count], 0].long(), torch.arange(count, device="cuda")) and (r.position[order[count:]] == -1).all()
    assert torch.equal(r.offsets.long(), torch.cat([key.new_zeros(1), torch.bincount(key, minlength=n + 1)[:n].cumsum(0)]))


def test_arguments_that_autograd_follows_are_warned_of(experts):
    r = experts.sort_by_expert(torch.zeros(4, 2, dtype=torch.int32, device="cuda"), 1)
    x, w, rows = torch.ones(4, 16, device="cuda", requires_grad=True), torch.ones(4, 2, device="cuda", requires_grad=True), torch.ones(8, 16, device="cuda")
    for call in (lambda: experts.dispatch(x, r), lambda: experts.combine(rows, w, r), lambda: experts.combine_backward(x, rows, w, r)):
        with pytest.warns(UserWarning, match="not recorded by autograd"):
            call()
        with torch.no_grad(), warnings.catch_warnings():
            warnings.simplefilter("error")
            call()

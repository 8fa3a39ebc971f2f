"""Log probabilities without a GPU: the oracle's pins, refusals of the C ABI and of LossHead, how calls are cut up."""
import contextlib
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import score_oracle
from paper_2502_16982_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2502_16982_amd", "csrc")
FAKE = 1 << 20


def test_oracle_against_autograd():
    g = torch.Generator().manual_seed(0)
    h = torch.randn(5, 7, generator=g, dtype=torch.float64, requires_grad=True)
    w = torch.randn(11, 7, generator=g, dtype=torch.float64, requires_grad=True)
    y = torch.tensor([3, -1, 0, 10, 5])
    dl, de = torch.randn(5, generator=g, dtype=torch.float64), torch.randn(5, generator=g, dtype=torch.float64)
    logp = torch.log_softmax(h @ w.T / 0.7, 1)
    entropy = -(logp.exp() * logp).sum(1)
    given = torch.where(y >= 0, logp.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
    (dl * given + de * entropy).sum().backward()
    got = score_oracle.scores(h.detach().numpy(), w.detach().numpy(), y.numpy(), 4, 0.7, dl.numpy(), de.numpy())
    for key, want in (("log_prob", given), ("entropy", entropy), ("lse", torch.logsumexp(h @ w.T / 0.7, 1)), ("d_hidden", h.grad), ("d_weight", w.grad),
                      ("top_log_prob", logp.topk(4).values)):
        assert np.allclose(got[key], want.detach().numpy(), rtol=1e-12, atol=1e-13), key
    assert np.array_equal(got["top_index"], logp.topk(4).indices.numpy())


def test_oracle_against_differences():
    rng = np.random.default_rng(1)
    h, w, y, dl, de = rng.standard_normal((3, 4)), rng.standard_normal((6, 4)), np.array([2, -1, 5]), rng.standard_normal(3), rng.standard_normal(3)

    def total(h, w):
        s = score_oracle.scores(h, w, y, 0, 1.3)
        return (dl * s["log_prob"] + de * s["entropy"]).sum()

    got = score_oracle.scores(h, w, y, 0, 1.3, dl, de)
    for x, d in ((h, got["d_hidden"]), (w, got["d_weight"])):
        for i in np.ndindex(x.shape):
            keep = x[i]
            x[i] = keep + 1e-5
            up = total(h, w)
            x[i] = keep - 1e-5
            down = total(h, w)
            x[i] = keep
            assert abs((up - down) / 2e-5 - d[i]) <= 1e-8


def test_oracle_orders_ties_by_index():
    s = score_oracle.scores(np.ones((1, 2)), np.array([[1.0, 0.0], [3.0, 0.0], [0.0, 1.0], [1.0, 2.0], [0.0, 0.0]]), None, 5)
    assert s["top_index"].tolist() == [[1, 3, 0, 2, 4]]


def head(tokens=4, vocab=100, width=16, dtype=1, hidden=FAKE, weight=FAKE, **over):
    h = binding.muon_head(hidden, weight, width, width, tokens, vocab, width, dtype, 0)
    for key, value in over.items():
        setattr(h, key, value)
    return h


def test_bytes():
    L, out = binding.lib(), C.c_size_t(0)
    call = lambda h, top=5, limit=0: L.muon_log_probs_bytes(C.byref(h) if h is not None else None, top, limit, C.byref(out))  # noqa: E731
    assert call(head()) == 0 and out.value > 0
    assert call(None) == -1 and L.muon_log_probs_bytes(C.byref(head()), 5, 0, None) == -1
    assert call(head(), top=-1) == call(head(), top=65) == call(head(vocab=4), top=5) == -1
    assert call(head(tokens=-1)) == call(head(vocab=0)) == call(head(vocab=(1 << 21) + 1)) == call(head(width=0)) == call(head(reserved=1)) == -1
    assert call(head(hidden_stride=15)) == call(head(weight_stride=15)) == -1
    assert call(head(dtype=2)) == -2
    assert call(head(hidden=FAKE + 1)) == call(head(weight=FAKE + 1)) == -7
    ask = lambda **kw: binding.muon_log_probs_bytes(head(**{k: v for k, v in kw.items() if k not in ("top", "limit")}), kw.get("top", 0), kw.get("limit", 0))  # noqa: E731
    for a, b in ((dict(tokens=5), dict(tokens=6)), (dict(vocab=1000), dict(vocab=1200)), (dict(top=0), dict(top=1)), (dict(tokens=8000), dict(tokens=90000)),
                 (dict(limit=1 << 20, tokens=90000, vocab=50000), dict(tokens=90000, vocab=50000))):
        assert ask(**a) <= ask(**b)
    assert ask(tokens=90000, vocab=50000, limit=1 << 27) <= 1 << 27


def test_refusals():
    L = binding.lib()
    need = binding.muon_log_probs_bytes(head(), 5)

    def call(h, targets=FAKE, size=8, top=5, tau=1.0, log_prob=FAKE, entropy=FAKE, lse=FAKE, rest=FAKE, index=FAKE, best=FAKE, kept=None, kept_bytes=0, ws=FAKE, nbytes=need):
        return L.muon_log_probs(C.byref(h), targets, size, top, tau, log_prob, entropy, lse, rest, index, best, kept, kept_bytes, ws, nbytes, None)

    h = head()
    for bad in (dict(size=2), dict(top=-1), dict(top=65), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")), dict(tau=float("inf")), dict(tau=1e-60),
                dict(log_prob=None), dict(targets=None), dict(entropy=None), dict(lse=None), dict(rest=None), dict(index=None), dict(best=None), dict(kept=FAKE, kept_bytes=1 << 30)):
        assert call(h, **bad) == -1, bad
    assert call(head(hidden=None)) == call(head(weight=None)) == -1
    assert call(h, ws=None) == call(h, nbytes=0) == call(h, nbytes=255) == -4
    for bad in (dict(targets=FAKE + 4), dict(log_prob=FAKE + 2), dict(entropy=FAKE + 2), dict(lse=FAKE + 2), dict(rest=FAKE + 2), dict(index=FAKE + 4),
                dict(best=FAKE + 2), dict(ws=FAKE + 128), dict(top=0, kept=FAKE + 128, kept_bytes=1 << 30)):
        assert call(h, **bad) == -7, bad
    room = binding.muon_log_probs_kept_bytes(h)
    assert room >= 4 * 256 * 2 and binding.muon_log_probs_kept_bytes(head(tokens=100, dtype=0)) >= 100 * 256 * 4
    assert binding.muon_log_probs_kept_bytes(head(dtype=0)) == binding.muon_log_probs_kept_bytes(head(width=15)) == 0
    assert L.muon_log_probs_kept_bytes(C.byref(h), None) == L.muon_log_probs_kept_bytes(None, C.byref(C.c_size_t())) == -1
    assert call(h, top=0, kept=FAKE, kept_bytes=room - 1) == -4
    assert call(head(tokens=0), ws=None) == 0

    back = binding.muon_head_workspace_bytes(head(), 1, 3)

    def backward(h, targets=FAKE, size=8, tau=1.0, lse=FAKE, rest=FAKE, entropy=FAKE, dl=FAKE, de=FAKE, kept=None, kept_bytes=0, dh=FAKE, dw=FAKE, ws=FAKE,
                 nbytes=back):
        return L.muon_log_probs_backward(C.byref(h), targets, size, tau, lse, rest, entropy, dl, de, kept, kept_bytes, dh, dw, ws, nbytes, None)

    for bad in (dict(size=1), dict(tau=0.0), dict(lse=None), dict(rest=None), dict(entropy=None), dict(dl=None), dict(targets=None), dict(targets=None, dl=None, de=None)):
        assert backward(h, **bad) == -1, bad
    assert backward(h, ws=None) == backward(h, nbytes=256) == backward(h, kept=FAKE, kept_bytes=room - 1) == -4
    assert backward(h, kept=FAKE + 128, kept_bytes=room) == -7
    for bad in (dict(targets=FAKE + 4), dict(lse=FAKE + 2), dict(rest=FAKE + 2), dict(entropy=FAKE + 2), dict(dl=FAKE + 2), dict(de=FAKE + 2), dict(dh=FAKE + 1),
                dict(dw=FAKE + 1), dict(ws=FAKE + 128)):
        assert backward(h, **bad) == -7, bad
    assert backward(h, dh=None, dw=None, ws=None, nbytes=0) == 0         # nothing is asked for
    assert backward(head(tokens=0), dw=None, ws=None) == 0


@pytest.fixture
def loss_head(monkeypatch):
    from paper_2502_16982_amd import losses
    calls = []
    monkeypatch.setattr(losses, "stream_handle", lambda device: 7)
    monkeypatch.setattr(losses, "on", lambda device: contextlib.nullcontext())
    monkeypatch.setattr(losses, "capturing", lambda: False)
    monkeypatch.setattr(losses, "current_stream", lambda device: None)
    monkeypatch.setattr(binding, "muon_log_probs", lambda *a: calls.append(a))
    monkeypatch.setattr(binding, "muon_log_probs_backward", lambda *a: calls.append(a))
    return losses.LossHead(4, 100, 16, device="cpu"), calls


def test_loss_head(loss_head):
    head, calls = loss_head
    h, w, y = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(100, 16, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    s = head.log_probs(h, w, y, top=3, temperature=0.5)
    assert s.top_index.shape == s.top_log_prob.shape == (4, 3) and s.top_index.dtype == torch.int64 and s.log_prob.shape == (4,)
    assert calls[-1][3:5] == (3, 0.5)
    bare = head.log_probs(h, w)
    assert bare.log_prob is None and bare.top_index is None and bare.entropy.shape == (4,) and calls[-1][1] == 0
    assert s.kept is None and bare.kept.numel() == binding.muon_log_probs_kept_bytes(calls[-1][0])       # alternatives, or what a backward call reads
    assert head.log_probs(h, w, keep=False).kept is None
    few = type(head)(4, 100, 16, device="cpu", max_workspace_bytes=600)
    assert few.log_probs(h, w).kept is None and few.log_probs(h, w, keep=True).kept is not None
    assert type(head)(4, 100, 16, device="cpu", gradients=False).log_probs(h, w).kept is None
    d = torch.ones(4)
    dh, dw = head.log_probs_backward(h, w, y, s, d, gradients=("weight",))
    assert dh is None and dw.shape == (100, 16)
    assert head.log_probs_backward(h, w, None, bare, None, d)[0].shape == (4, 16)
    for call in (lambda: head.log_probs(h, w, y[:3]), lambda: head.log_probs(h, w, y.float()), lambda: head.log_probs(h, w, top=65),
                 lambda: head.log_probs(h, w, top=-1), lambda: head.log_probs_backward(h, w, y, s, None, d), lambda: head.log_probs_backward(h, w, None, s, d),
                 lambda: head.log_probs_backward(h, w, None, s, None), lambda: head.log_probs_backward(h, w, y, s, d[:3]),
                 lambda: head.log_probs_backward(h, w, y, s, d.double()), lambda: head.log_probs_backward(h[:3], w, y[:3], s, d[:3]),
                 lambda: head.log_probs_backward(h, w, y, s._replace(kept=bare.kept[:-1]), d)):
        with pytest.raises(binding.MuonError):
            call()
    with pytest.warns(UserWarning, match="not recorded by autograd"):
        head.log_probs(h.requires_grad_(), w, y)


def test_plans(tmp_path):
    exe = str(tmp_path / "score_plan")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", f"-I{CSRC}",
                    os.path.join(ROOT, "tests", "score_plan_main.cpp"), os.path.join(CSRC, "score_plan.cpp"), os.path.join(CSRC, "head_plan.cpp"), "-o", exe],
                   check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and "ok" in out.stdout, out.stdout + out.stderr


def test_scores_of_another_device_are_refused(loss_head):
    """Each tensor of the scores whose address goes to the library has to be where the workspace is."""
    head, calls = loss_head
    h, w, y = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(100, 16, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    s, d = head.log_probs(h, w, y), torch.ones(4)
    head.log_probs_backward(h, w, y, s, d, d)
    count = len(calls)
    for name in ("lse", "lse_rest", "entropy", "kept"):
        with pytest.raises(binding.MuonError, match="is on meta|another call"):
            head.log_probs_backward(h, w, y, s._replace(**{name: getattr(s, name).to("meta")}), d, d)
    assert len(calls) == count


def test_what_is_kept_by_default_is_bounded(loss_head, monkeypatch):
    """Without a limit of the LossHead's own the kept powers of a long batch would outgrow everything else."""
    from paper_2502_16982_amd import losses
    head, calls = loss_head
    assert losses.KEEP_BYTES == 8 << 30
    h, w = torch.zeros(40000, 8, dtype=torch.bfloat16), torch.zeros(131072, 8, dtype=torch.bfloat16)
    assert 40000 * 131072 * 2 > losses.KEEP_BYTES
    assert head.log_probs(h, w).kept is None and calls[-1][11] == 0
    h, w = h[:20], w[:1000]
    need = 20 * 1024 * 2 + (20 * 8 * 4 + 255) // 256 * 256
    monkeypatch.setattr(losses, "KEEP_BYTES", need - 1)
    assert head.log_probs(h, w).kept is None and calls[-1][11] == 0
    kept = head.log_probs(h, w, keep=True).kept
    assert kept.numel() == need and calls[-1][11:13] == (kept.data_ptr(), need)
    assert losses.LossHead(20, 1000, 8, device="cpu", max_workspace_bytes=1 << 24).log_probs(h, w).kept.numel() == need      # the limit given counts instead
    assert losses.LossHead(20, 1000, 8, device="cpu", max_workspace_bytes=need - 1).log_probs(h, w).kept is None
    monkeypatch.setattr(losses, "KEEP_BYTES", need)
    assert head.log_probs(h, w).kept.numel() == need

"""Pins of the oracles of the head's losses and of the experts' dispatch: hand-worked values, differences, symmetries (CPU)."""
import numpy as np
import pytest

from oracle import experts_oracle as ex
from oracle import head_oracle as ho


def test_cross_entropy_hand_worked():
    # two logits (0, log 3): p = (1/4, 3/4)
    h, w = np.array([[1.0]]), np.array([[0.0], [np.log(3.0)]])
    r = ho.head_loss(h, w, targets=[1])
    assert np.isclose(r["loss"][0], -np.log(0.75)) and np.isclose(r["lse"][0], np.log(4.0))
    assert np.allclose(r["d_logits"], [[0.25, -0.25]])
    assert np.allclose(r["d_hidden"], [[-0.25 * np.log(3.0)]]) and np.allclose(r["d_weight"], [[0.25], [-0.25]])


def test_distillation_of_the_students_own_softmax_is_zero():
    g = np.random.default_rng(1)
    h, w = g.normal(size=(4, 6)), g.normal(size=(9, 6))
    index = np.tile(np.arange(9), (4, 1))
    r = ho.head_loss(h, w, index=index, teacher=h @ w.T, tau=1.7)
    assert np.allclose(r["loss"], 0.0, atol=1e-12) and np.allclose(r["d_logits"], 0.0, atol=1e-12)


def test_distillation_with_one_entry_is_cross_entropy():
    g = np.random.default_rng(2)
    h, w, y = g.normal(size=(5, 6)), g.normal(size=(9, 6)), g.integers(0, 9, 5)
    a = ho.head_loss(h, w, targets=y)
    b = ho.head_loss(h, w, index=y[:, None], teacher=g.normal(size=(5, 1)))
    for k in a:
        assert np.allclose(a[k], b[k])


def test_an_entry_that_occurs_twice_counts_twice():
    g = np.random.default_rng(3)
    h, w = g.normal(size=(1, 6)), g.normal(size=(9, 6))
    a = ho.head_loss(h, w, index=np.array([[2, 2, 5]]), teacher=np.array([[0.0, 0.0, 1.0]]))
    p = np.exp(w @ h[0]) / np.exp(w @ h[0]).sum()
    q = np.array([1.0, 1.0, np.e]) / (2 + np.e)
    assert np.isclose(a["loss"][0], (q * (np.log(q) - np.log(p[[2, 2, 5]]))).sum())
    assert np.isclose(a["d_logits"][0, 2], p[2] - 2 * q[0])


def test_tokens_without_target_or_scale():
    g = np.random.default_rng(4)
    h, w = g.normal(size=(4, 6)), g.normal(size=(9, 6))
    h[1], h[2] = np.nan, np.inf
    r = ho.head_loss(h, w, targets=[3, -100, 4, 9], scale=[1.0, 1.0, 0.0, 1.0])
    assert r["loss"][1] == 0.0 and np.isnan(r["loss"][3])
    assert np.all(r["d_logits"][1:] == 0.0) and np.all(np.isfinite(r["d_weight"]))
    r = ho.head_loss(h[:1], w, index=np.array([[-1, 3]]), teacher=np.array([[np.nan, -np.inf]]))
    assert r["loss"][0] == 0.0 and np.all(r["d_logits"] == 0.0)


@pytest.mark.parametrize("kind", ["ce", "distill"])
def test_gradients_against_differences(kind):
    g = np.random.default_rng(5)
    h, w, scale = g.normal(size=(3, 5)), g.normal(size=(7, 5)), g.normal(size=3)
    more = dict(targets=[2, -1, 6]) if kind == "ce" else dict(index=np.array([[1, 4, 4], [0, -1, 2], [6, 5, 3]]),
                                                            teacher=g.normal(size=(3, 3)), tau=1.3)
    r = ho.head_loss(h, w, scale=scale, **more)
    for x, d in ((h, r["d_hidden"]), (w, r["d_weight"])):
        for at in np.ndindex(x.shape):
            keep, step = x[at], 1e-6
            x[at] = keep + step
            up = (scale * ho.head_loss(h, w, scale=scale, **more)["loss"]).sum()
            x[at] = keep - step
            down = (scale * ho.head_loss(h, w, scale=scale, **more)["loss"]).sum()
            x[at] = keep
            assert abs((up - down) / (2 * step) - d[at]) < 1e-7


def test_sort_is_stable_and_drops():
    expert = np.array([[1, 0], [0, -1], [1, 7], [0, 1]])
    position, source, offsets = ex.sort_pairs(expert, 2)
    assert offsets.tolist() == [0, 3, 6]
    assert source.tolist() == [1, 2, 6, 0, 4, 7, -1, -1]
    assert position.tolist() == [[3, 0], [1, -1], [4, -1], [2, 5]]


def test_dispatch_and_combine_are_adjoint():
    g = np.random.default_rng(6)
    position, _, _ = ex.sort_pairs(g.integers(-1, 5, (7, 3)), 5)
    x, rows, w, d = g.normal(size=(7, 4)), g.normal(size=(21, 4)), g.normal(size=(7, 3)), g.normal(size=(7, 4))
    kept = np.zeros(21, bool)
    kept[position[position >= 0]] = True
    rows[~kept] = 0.0
    assert np.isclose((ex.dispatch(x, position) * rows).sum(), (x * ex.combine(rows, None, position)).sum())
    d_rows, d_w = ex.combine_backward(d, rows, w, position)
    out = (ex.combine(rows, w, position) * d).sum()
    assert np.isclose((d_rows * rows).sum(), out) and np.isclose((d_w * w).sum(), out)       # linear in each

"""Pins of the float64 definitions of the operators around the projections
(oracle/step_oracle.py): hand-worked values, identities, gradients against
differences, and the law that verified drafts follow the target."""
import math

import numpy as np
import pytest

from oracle import step_oracle as so

RNG = lambda *seed: np.random.default_rng([7, *seed])  # noqa: E731


def test_fused_by_hand():
    Q = np.array([[2, -3, 1], [0, 5, -127]], np.int8)
    scale = np.array([0.5, 0.25], np.float32)
    x = np.array([[1.0, 2.0, 4.0]], np.float32)
    bias = np.array([1.0, 100.0], np.float32)
    # row 0: 2 - 6 + 4 = 0; row 1: 10 - 508 = -498 -> -124.5
    assert so.fused_forward(Q, scale, x, bias).tolist() == [[1.0, -24.5]]
    assert so.fused_forward(Q, scale, x, bias, "relu", np.array([[3.0, 4.0]])).tolist() == [[4.0, 4.0]]
    dx, dbias, _ = so.fused_backward(Q, scale, np.array([[4.0, 8.0]]), np.array([[1.0, -24.5]]), "relu")
    assert dx.tolist() == [[4.0, -6.0, 2.0]] and dbias.tolist() == [4.0, 0.0]


@pytest.mark.parametrize("kind", ["none", "relu", "gelu", "silu"])
def test_slopes_are_the_differences(kind):
    z = np.linspace(-9, 9, 401) + 0.013  # no point within a step of the kink
    h = 1e-5
    diff = (so.act(z + h, kind) - so.act(z - h, kind)) / (2 * h)
    assert np.abs(diff - so.act_slope(z, kind)).max() < 1e-9  # truncation h^2 / 6 * |act'''| and rounding 1e-16 * 9 / h


def test_gelu_values():
    # Phi(1) = 0.841344746068543, Phi(-3) = 0.001349898031630
    z = np.array([1.0, -3.0, 0.0])
    assert np.allclose(so.act(z, "gelu"), [0.841344746068543, -0.00404969409489, 0.0], rtol=1e-11, atol=0)


@pytest.mark.parametrize("kind", ["none", "relu", "gelu", "silu"])
def test_fused_gradient_is_the_difference(kind):
    r = RNG(1)
    Q = r.integers(-127, 128, (9, 11)).astype(np.int8)
    scale, bias = r.uniform(0.001, 0.01, 9), r.normal(size=9)
    x, dy, v, vb = r.normal(size=(5, 11)), r.normal(size=(5, 9)), r.normal(size=(5, 11)), r.normal(size=9)
    f = lambda t: (so.fused_forward(Q, scale, x + t * v, bias + t * vb, kind) * dy).sum()  # noqa: E731
    h = 1e-6
    dx, dbias, _ = so.fused_backward(Q, scale, dy, so.fused_pre(Q, scale, x, bias), kind)
    want = (dx * v).sum() + (dbias * vb).sum()
    assert abs((f(h) - f(-h)) / (2 * h) - want) < 1e-7 * max(1.0, abs(want))


def test_embedding_and_its_gradient_are_adjoint():
    r = RNG(2)
    table, ids = r.normal(size=(7, 5)), np.array([3, -1, 0, 3, 7, 6, 3])
    grad = r.normal(size=(7, 5))
    lhs = (so.embed_forward(table, ids, 1.5) * grad).sum()
    assert math.isclose(lhs, (table * so.embed_backward(grad, ids, 7, 1.5)).sum(), rel_tol=1e-12)
    assert (so.embed_forward(table, ids, 1.5)[[1, 4]] == 0).all()
    assert (so.embed_backward(grad, ids, 7, 1.0)[3] == (grad[0] + grad[3]) + grad[6]).all()


def test_probabilities_special_rows():
    inf = np.inf
    assert so.probabilities(np.array([-inf, np.nan, -inf]), 1.0).tolist() == [0, 0, 0]
    assert so.probabilities(np.array([1.0, inf, np.nan, inf]), 0.5).tolist() == [0, 0.5, 0, 0.5]
    assert so.probabilities(np.array([1.0, 3.0, 3.0]), 0.0).tolist() == [0, 1, 0]
    p = so.probabilities(np.array([0.0, math.log(3.0)]), 1.0)
    assert np.allclose(p, [0.25, 0.75], rtol=1e-15)


def test_draft_by_hand():
    """Two drafts over three tokens: the first accepted (0.5 * 0.5 < 0.6), the
    second refused (0.9 * 0.8 >= 0.2); residual (0.4 - 0.1, 0, 0.4 - 0.1) raced with
    noise (2, 1, 1): token 2."""
    p = np.log(np.array([[[0.6, 0.3, 0.1], [0.4, 0.2, 0.4], [1.0, 1.0, 1.0]]]))
    q = np.log(np.array([[[0.5, 0.4, 0.1], [0.1, 0.8, 0.1]]]))
    out = so.draft_verify(p, q, np.array([[0, 1]]), np.array([[0.5, 0.9]]), np.array([[2.0, 1.0, 1.0]]))
    assert out[0].tolist() == [[0, 2, -1]] and out[1].tolist() == [1]
    assert np.allclose(out[2], [[1.0, 0.25]]) and np.allclose(out[3], [[0.6, 0.4, 0.0]])


def test_verified_drafts_follow_the_target():
    """The first emitted token's law is the target's, whatever the draft's: 40,000
    draws, each frequency within 5 standard deviations."""
    r = RNG(3)
    n, V = 40000, 4
    pt, qt = np.array([0.5, 0.2, 0.2, 0.1]), np.array([0.1, 0.6, 0.1, 0.2])
    target = np.broadcast_to(np.log(np.stack([pt, pt])), (n, 2, V))
    draft = np.broadcast_to(np.log(qt)[None], (n, 1, V))
    drafts = r.choice(V, size=(n, 1), p=qt)
    tokens = so.draft_verify(target, draft, drafts, r.random((n, 1)), r.exponential(size=(n, V)))[0]
    freq = np.bincount(tokens[:, 0], minlength=V) / n
    assert (np.abs(freq - pt) < 5 * np.sqrt(pt * (1 - pt) / n)).all(), freq


@pytest.mark.parametrize("mistake", ["keep_draft", "no_subtract", "le"])
def test_planted_mistakes_show(mistake):
    """The law above tells the definition from near misses (the mistakes are planted here, in the oracle's arithmetic)."""
    r = RNG(4)
    n = 40000
    pt, qt = np.array([0.5, 0.2, 0.2, 0.1]), np.array([0.1, 0.6, 0.1, 0.2])
    d = r.choice(4, size=n, p=qt)
    u = r.random(n)
    if mistake == "le":  # the comparison the other way round
        ok = u * qt[d] >= pt[d]
    else:
        ok = u * qt[d] < pt[d]
    res = pt if mistake == "no_subtract" else np.maximum(pt - qt, 0)
    second = d if mistake == "keep_draft" else (res[None] / r.exponential(size=(n, 4))).argmax(axis=1)
    freq = np.bincount(np.where(ok, d, second), minlength=4) / n
    assert (np.abs(freq - pt) > 5 * np.sqrt(pt * (1 - pt) / n)).any()

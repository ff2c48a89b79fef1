"""Pins of the language-model oracle: closed forms, differences, adjointness."""
import numpy as np
import pytest

from oracle import text as OT


def test_lookup_and_gradient_are_adjoint():
    """<G, embed(E)> = <E, embed_grad(G)>: the gradient is the transpose of the (linear) lookup."""
    rng = np.random.default_rng(0)
    n, V, h, T = 3, 7, 5, 11
    E, G = rng.standard_normal((n, V, h)), rng.standard_normal((n, T, h))
    tokens = rng.integers(-1, V + 1, (n, T))
    left = (G * OT.embed(E, tokens, 1.5)).sum()
    dE, size, terms = OT.embed_grad(G, tokens, V, 1.5)
    assert np.isclose(left, (E * dE).sum(), rtol=1e-12)
    assert terms.sum() == ((tokens >= 0) & (tokens < V)).sum() and (size >= np.abs(dE) - 1e-12).all()
    again, _, _ = OT.embed_grad(G, tokens, V, 1.5, old=dE)
    assert np.allclose(again, 2 * dE, rtol=1e-12)


@pytest.mark.parametrize("temperature,hard", [(1.0, 0.0), (2.0, 0.3), (0.5, 1.0)])
def test_distillation_gradient_against_differences(temperature, hard):
    rng = np.random.default_rng(1)
    V, K = 9, 4
    s, u = rng.standard_normal(V), rng.standard_normal(K)
    ids = np.array([2, 7, 2, V])                                     # one place twice, one outside
    _, grad, _ = OT.distill_row(s, u, ids, temperature, hard, 5, 0.7)
    for v in range(V):
        step = np.zeros(V)
        step[v] = 1e-5
        up, down = (OT.distill_row(x, u, ids, temperature, hard, 5, 0.7)[0] for x in (s + step, s - step))
        assert abs((up - down) / 2e-5 - grad[v]) <= 1e-8


def test_distillation_closed_forms():
    # a student that agrees with the teacher on all of the vocabulary: no loss, no gradient
    s = np.array([0.3, -1.0, 2.0])
    loss, grad, _ = OT.distill_row(s, s + 4.0, np.arange(3), 2.0, 0.0, None, 1.0)
    assert abs(loss) < 1e-14 and np.abs(grad).max() < 1e-14
    # uniform student, one certain entry: tau^2 log V
    loss, grad, _ = OT.distill_row(np.zeros(8), np.array([3.0]), np.array([5]), 3.0, 0.0, None, 1.0)
    assert np.isclose(loss, 9 * np.log(8)) and np.isclose(grad[5], 3 * (1 / 8 - 1)) and np.isclose(grad[0], 3 / 8)
    # cross entropy alone; empty rows
    loss, _, _ = OT.distill_row(np.zeros(8), [], [], 1.0, 1.0, 2, 1.0)
    assert np.isclose(loss, np.log(8))
    assert OT.distill_row(np.full(4, -np.inf), np.array([1.0]), np.array([1]), 1.0, 0.0, None, 1.0)[0] == 0
    assert OT.distill_row(np.zeros(4), np.array([1.0]), np.array([-1]), 1.0, 0.0, None, 1.0)[0] == 0


def test_top_logits_by_hand():
    rows = np.array([[1.0, 3.0, -np.inf, 3.0, 2.0], [-np.inf] * 4 + [0.0], [np.nan, np.inf, 0.0, -0.0, np.nan]])
    values, ids = OT.top_logits(rows, 3)
    assert ids.tolist() == [[1, 3, 4], [4, -1, -1], [0, 4, 1]]
    assert values[0].tolist() == [3.0, 3.0, 2.0] and values[1].tolist() == [0.0, -np.inf, -np.inf]
    assert OT.top_logits(rows, 5)[1][2].tolist() == [0, 4, 1, 2, 3]

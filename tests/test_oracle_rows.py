"""Pins of the 64-bit definitions of layer norm, embedding and distillation: gradients against differences, and what they say by hand."""
import numpy as np
import pytest

from oracle import rows_ref as ref


def _difference(f, x, h=1e-6):
    """Gradient of f at x by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + h
        up = f()
        x[i] = keep - h
        g[i] = (up - f()) / (2 * h)
        x[i] = keep
    return g


@pytest.mark.parametrize("d", [1, 2, 5, 8])
def test_norm_gradients_are_differences(d):
    rng = np.random.default_rng(d)
    x, g = rng.normal(size=(4, d)), rng.normal(size=(4, d))
    gamma, beta = 1 + rng.normal(size=d), rng.normal(size=d)
    eps = 1e-2
    y, mean, rstd = ref.norm_fwd(x, gamma, beta, eps)
    f = lambda: (ref.norm_fwd(x, gamma, beta, eps)[0] * g).sum()
    for got, at in zip(ref.norm_bwd(x, g, gamma, mean, rstd), (x, gamma, beta)):
        assert np.allclose(got, _difference(f, at), atol=1e-7, rtol=1e-7)
    xh = (y - beta) / gamma
    assert np.allclose(xh.mean(1), 0) and np.all((xh ** 2).mean(1) <= 1)


def test_embedding_gradient_is_a_difference():
    rng = np.random.default_rng(0)
    table, tokens = rng.normal(size=(5, 3)), np.array([4, 0, 2, 2, 7, -1, 2, 0])
    g = rng.normal(size=(8, 3))
    f = lambda: (ref.embed_fwd(tokens, table, 1.5, 0) * g).sum()
    got, mag = ref.embed_bwd(tokens, g, 1.5, 0, 5)
    assert np.allclose(got, _difference(f, table), atol=1e-8)
    assert np.all(got[[0, 1, 3]] == 0) and np.allclose(got[2], 1.5 * (g[2] + g[3] + g[6])) and np.all(mag >= np.abs(got) - 1e-12)
    keys, index = ref.token_order(tokens, 0, 5)
    assert keys.tolist() == [2, 2, 2, 4, 5, 5, 5, 5] and index.tolist() == [2, 3, 6, 0, 1, 4, 5, 7]


@pytest.mark.parametrize("hard", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("T", [1.0, 2.5])
def test_distillation_gradient_is_a_difference(hard, T):
    rng = np.random.default_rng(3)
    z, logits = rng.normal(size=(5, 6)), rng.normal(size=(5, 3))
    ids = np.array([[0, 3, 5], [1, 1, 2], [4, -1, -1], [-1, -1, -1], [2, 9, 0]])   # a class twice, fewer entries, none, one outside
    labels, w = np.array([3, -1, 0, 5, 7]), np.array([1.0, 0.5, 2.0, 1.0, 0.3])
    loss, g = ref.distill(z, ids, logits, T, hard, labels, w)
    f = lambda: (ref.distill(z, ids, logits, T, hard, labels, w)[0] * w).sum()
    assert np.allclose(g, _difference(f, z), atol=1e-7)
    assert np.allclose(g.sum(1), 0, atol=1e-12) and np.all(loss >= -1e-12)


def test_distillation_by_hand():
    # a student that agrees with the teacher over all classes has nothing to learn; a row of weight 0 is not looked at
    z = np.array([[0.0, 1.0, 2.0], [np.nan, np.inf, 0.0]])
    ids, logits = np.array([[0, 1, 2]] * 2), np.array([[5.0, 6.0, 7.0]] * 2)
    loss, g = ref.distill(z, ids, logits, 2.0, 0.0, None, np.array([1.0, 0.0]))
    assert np.allclose(loss, 0) and np.allclose(g, 0)
    # all of the teacher's weight on one class: cross-entropy
    loss, g = ref.distill(z[:1], np.array([[2, -1]]), np.array([[3.0, 9.0]]), 1.0, 0.0, None, np.ones(1))
    assert np.isclose(loss[0], np.log(1 + np.exp(-1) + np.exp(-2)))
    # a logit of -inf is no entry
    same, _ = ref.distill(z[:1], np.array([[2, 0]]), np.array([[3.0, -np.inf]]), 1.0, 0.0, None, np.ones(1))
    assert same[0] == loss[0]

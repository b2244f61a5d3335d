"""The fp64 definitions of the operators around the layers, pinned by hand-worked cases and by differences."""
import numpy as np
import pytest

from oracle import tokens as tok


def test_embedding_by_hand():
    table = [[1.0, 2.0], [3.0, 4.0], [5.0, 6.0]]
    np.testing.assert_array_equal(tok.embed(table, [2, -1, 0, 3, 2], 0.5), [[2.5, 0, 0.5, 0, 2.5], [3, 0, 1, 0, 3]])
    G = np.array([[1.0, 10, 100, 1000, 10000], [2.0, 20, 200, 2000, 20000]])
    np.testing.assert_array_equal(tok.embed_gradient(3, [2, -1, 0, 3, 2], G, 0.5), [[50, 100], [0, 0], [5000.5, 10001]])


def test_norm_by_hand():
    Y, rstd = tok.norm([[3.0, 0.0], [4.0, 0.0]], [1.0, 2.0], 0.25)
    np.testing.assert_allclose(rstd, [1 / np.sqrt(12.75), 2.0])
    np.testing.assert_allclose(Y, [[3 / np.sqrt(12.75), 0], [8 / np.sqrt(12.75), 0]])


def test_log_prob_by_hand():
    # softmax of (log 1, log 2, log 5) is (1, 2, 5) / 8; the second column is masked but for its first row
    x = np.array([[0.0, 7.0, -np.inf], [np.log(2), -np.inf, -np.inf], [np.log(5), -np.inf, -np.inf]])
    logp, H, top_logp, top_ids = tok.log_prob(x, [1, -1, 2], 2)
    p = np.array([1, 2, 5]) / 8
    np.testing.assert_allclose(logp, [np.log(0.25), 0, -np.inf])
    np.testing.assert_allclose(H, [-np.sum(p * np.log(p)), 0, 0], atol=1e-15)
    np.testing.assert_array_equal(top_ids, [[2, 0, -1], [1, -1, -1]])
    np.testing.assert_allclose(top_logp, [[np.log(0.625), 0, -np.inf], [np.log(0.25), -np.inf, -np.inf]])
    dx = tok.log_prob_gradient(x, [1, -1, 2], [1.0, 5.0, 3.0], None)
    np.testing.assert_allclose(dx, [[-1 / 8, 0, 0], [3 / 4, 0, 0], [-5 / 8, 0, 0]])


def test_ties_go_to_the_lower_row():
    _, _, _, ids = tok.log_prob(np.array([[1.0], [2.0], [2.0], [1.0], [np.nan]]), None, 4)
    np.testing.assert_array_equal(ids[:, 0], [1, 2, 0, 3])


def _differences(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        hi, lo = x.copy(), x.copy()
        hi[i] += h
        lo[i] -= h
        g[i] = (f(hi) - f(lo)) / (2 * h)
    return g


@pytest.mark.parametrize("seed", range(3))
def test_gradients_by_differences(seed):
    """Central differences with h = 1e-6 in fp64: 1e-12 from the third derivative and 1e-10 from rounding, on values near 1."""
    r = np.random.default_rng(seed)
    vocab, d, m = 6, 5, 4
    ids = r.integers(-1, vocab, m)
    G = r.normal(size=(d, m))
    table = r.normal(size=(vocab, d))
    np.testing.assert_allclose(tok.embed_gradient(vocab, ids, G, 1.7), _differences(lambda t: np.sum(G * tok.embed(t, ids, 1.7)), table), atol=1e-8)
    S, w, dS, eps = r.normal(size=(d, m)), r.normal(size=d), r.normal(size=(d, m)), 0.1
    dX, dw = tok.norm_gradient(G, S, w, eps, dS)
    np.testing.assert_allclose(dX, _differences(lambda s: np.sum(G * tok.norm(s, w, eps)[0]) + np.sum(dS * s), S), atol=1e-8)
    np.testing.assert_allclose(dw, _differences(lambda v: np.sum(G * tok.norm(S, v, eps)[0]), w), atol=1e-8)
    x, gl, ge = r.normal(size=(vocab, m)), r.normal(size=m), r.normal(size=m)

    def loss(x):
        logp, H, _, _ = tok.log_prob(x, ids)
        return np.sum(gl * logp) + np.sum(ge * H)

    np.testing.assert_allclose(tok.log_prob_gradient(x, ids, gl, ge), _differences(loss, x), atol=1e-8)


def test_clipping_by_hand():
    assert tok.grad_clip([[3.0], [4.0]], 1.0) == (5.0, 0.2)
    assert tok.grad_clip([[3.0], [4.0]], 5.0) == (5.0, 1.0)
    assert tok.grad_clip([[np.inf]], 1.0) == (np.inf, 1.0)

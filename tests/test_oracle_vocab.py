"""Pins of oracle/vocab.py: closed forms, a brute-force ranking, and central differences for every gradient."""
import numpy as np

from oracle import vocab as O


def test_uniform_and_two_valued_rows():
    x = np.zeros((1, 7))
    logp, entropy, stats, ids, alt = O.token_logprobs(x, [3], 0.5, 4)
    assert np.isclose(logp[0], -np.log(7)) and np.isclose(entropy[0], np.log(7))
    assert stats[0, 0] == 0 and np.isclose(stats[0, 1], np.log(7))
    assert ids.tolist() == [[0, 1, 2, 3]] and np.allclose(alt, -np.log(7))
    # p = 3/4 and 1/4 at temperature 2: values 2 ln 3 apart
    x = np.array([[0.0, 2 * np.log(3.0), -np.inf]])
    logp, entropy, _, ids, _ = O.token_logprobs(x, [1], 2.0, 3)
    assert np.isclose(logp[0], np.log(0.75)) and ids.tolist() == [[1, 0, 2]]
    assert np.isclose(entropy[0], -0.75 * np.log(0.75) - 0.25 * np.log(0.25))


def test_rows_without_a_distribution():
    x = np.array([[-np.inf] * 3, [np.nan, 1.0, 0.0], [np.inf, 1.0, 0.0]])
    logp, entropy, stats, ids, _ = O.token_logprobs(x, [1, 1, 1], 1.0, 3)
    assert logp[0] == -np.inf and entropy[0] == 0 and (stats[0] == -np.inf).all()
    assert np.isnan(logp[1:]).all() and np.isnan(entropy[1:]).all()
    assert ids.tolist() == [[0, 1, 2], [1, 2, 0], [0, 1, 2]]
    g = O.token_logprobs_grad(x, [1, 1, 1], 1.0, [1.0, 1.0, 0.0])
    assert (g[0] == 0).all() and np.isnan(g[1]).all() and (g[2] == 0).all()
    assert O.token_logprobs(x, [-1, 5, -1], 1.0)[0].tolist() == [0.0, 0.0, 0.0]


def _differences(f, x, step=1e-6):
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += step
        down[i] -= step
        out[i] = (f(up) - f(down)) / (2 * step)
    return out


def test_logits_gradient_against_differences():
    rng = np.random.default_rng(3)
    x = rng.normal(0, 2, (3, 11))
    t, g, h = [4, -1, 0], rng.normal(size=3), rng.normal(size=3)

    def f(x):
        logp, entropy, *_ = O.token_logprobs(x, t, 0.8)
        return float(g @ logp + h @ entropy)

    assert np.allclose(O.token_logprobs_grad(x, t, 0.8, g, h), _differences(f, x), atol=1e-8)


def test_head_gradients_against_differences():
    rng = np.random.default_rng(4)
    a, w = rng.normal(size=(3, 5)), rng.normal(size=(7, 5))
    t, g, h = [6, 2, -1], rng.normal(size=3), rng.normal(size=3)

    def f(a, w):
        logp, entropy, _ = O.head_logprobs(a, w, t, 1.3)
        return float(g @ logp + h @ entropy)

    da, dw, _ = O.head_logprobs_grad(a, w, t, 1.3, g, h)
    assert np.allclose(da, _differences(lambda v: f(v, w), a), atol=1e-8)
    assert np.allclose(dw, _differences(lambda v: f(a, v), w), atol=1e-8)


def test_embedding_and_its_gradient():
    rng = np.random.default_rng(5)
    table, ids = rng.normal(size=(4, 3)), [2, 0, 2, -1, 4]
    dy, base = rng.normal(size=(5, 3)), rng.normal(size=(4, 3))
    assert np.allclose(O.embed(table, ids, 2.0), [2 * table[2], 2 * table[0], 2 * table[2], [0] * 3, [0] * 3])
    f = lambda e: float(np.sum(dy * O.embed(e, ids, 2.0)) + np.sum(base * e))  # noqa: E731
    assert np.allclose(O.embed_grad(dy, ids, 4, 2.0, base), _differences(f, table), atol=1e-8)

"""The oracle of the token log probabilities: closed forms, brute force, and its gradient against differences.  CPU only."""
import numpy as np

from oracle import logprobs


def test_closed_forms():
    x = np.zeros((7, 2))
    lp = logprobs.log_probs(x)
    assert np.allclose(lp, -np.log(7)) and np.allclose(logprobs.entropy(lp), np.log(7))
    x = np.log(np.array([[1.0], [2.0], [5.0]]))
    lp = logprobs.log_probs(x)
    assert np.allclose(np.exp(lp[:, 0]), [1 / 8, 2 / 8, 5 / 8])
    assert np.allclose(logprobs.entropy(lp), -(1 / 8 * np.log(1 / 8) + 2 / 8 * np.log(2 / 8) + 5 / 8 * np.log(5 / 8)))
    x = np.array([[1.0, -np.inf], [-np.inf, -np.inf]])
    lp = logprobs.log_probs(x)
    assert lp[0, 0] == 0 and np.isneginf(lp[1, 0]) and np.isneginf(lp[:, 1]).all()
    assert np.array_equal(logprobs.entropy(lp), [0, 0])
    assert np.array_equal(logprobs.of_tokens(lp, [-1, 5])[:1], [0]) and np.isnan(logprobs.of_tokens(lp, [-1, 5])[1])


def test_top_words():
    x = np.array([[1.0, -np.inf], [3.0, -np.inf], [3.0, 0.0], [2.0, np.nan]])
    assert np.array_equal(logprobs.top(x, 3), [[1, 2], [2, -1], [3, -1]])


def test_gradient_against_differences():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((11, 4)) * 2
    x[2, 1] = -np.inf
    tokens = np.array([3, 0, -1, 10])
    gl, gh = rng.standard_normal(4), rng.standard_normal(4)

    def loss(x):
        lp = logprobs.log_probs(x)
        return (gl * logprobs.of_tokens(lp, tokens) + gh * logprobs.entropy(lp)).sum()

    got = logprobs.grad(x, tokens, gl, gh)
    h = 1e-5
    for v in range(11):
        for q in range(4):
            if np.isneginf(x[v, q]):
                assert got[v, q] == 0
                continue
            up, down = x.copy(), x.copy()
            up[v, q] += h
            down[v, q] -= h
            assert abs((loss(up) - loss(down)) / (2 * h) - got[v, q]) < 1e-8  # third derivatives times h^2 / 6, and 2^-53 / h
    # the whole gradient of a column sums to zero: adding a number to all logits changes nothing
    assert np.allclose(got.sum(axis=0), 0, atol=1e-12)

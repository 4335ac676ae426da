"""Pins of the oracle of filtered sampling: worked examples and what follows from the definitions."""
import numpy as np

from oracle import filtered_sampling as OF

X = np.log([0.1, 0.4, 0.2, 0.4, 0.05])                     # order: 1, 3, 2, 0, 4; shares of 1.15


def test_each_filter():
    keep = lambda **kw: OF.kept_tokens(X, **kw).tolist()
    assert keep() == [1, 3, 2, 0, 4]
    assert [keep(top_k=k) for k in (1, 2, 4, 5, 9, -3)] == [[1], [1, 3], [1, 3, 2, 0], [1, 3, 2, 0, 4], [1, 3, 2, 0, 4], [1, 3, 2, 0, 4]]
    # sums before the places: 0, 0.4, 0.8, 1.0, 1.1 of 1.15
    assert [keep(top_p=p) for p in (0.3, 0.35, 0.69, 0.7, 0.86, 0.87, 1.0, 0.0, -1.0)] == [
        [1], [1, 3], [1, 3], [1, 3, 2], [1, 3, 2], [1, 3, 2, 0], [1, 3, 2, 0, 4], [1], [1]]
    assert [keep(min_p=m) for m in (0.12, 0.2, 0.3, 0.6, 1.0, 1.5)] == [[1, 3, 2, 0, 4], [1, 3, 2, 0], [1, 3, 2], [1, 3], [1, 3], [1]]
    # mass of the first two alone: 0.4 of 0.8 is not below half of it
    assert keep(top_k=2, top_p=0.5) == [1] and keep(top_k=2, top_p=0.51) == [1, 3]
    assert keep(top_k=4, top_p=0.8, min_p=0.6) == [1, 3]
    assert keep(temperature=0.0) == [1] and keep(temperature=np.inf, top_p=0.5) == [1, 3, 2]


def test_draws():
    assert [OF.sample(X, u, top_k=3)[0] for u in (0.0, 0.39, 0.41, 0.59, 0.61, 0.999)] == [1, 1, 2, 2, 3, 3]
    token, logp, n = OF.sample(X, 0.5, top_k=3)
    assert n == 3 and np.isclose(logp, np.log(0.2 / 1.0))
    assert OF.sample(X, 0.9, temperature=0.0) == (1, 0.0, 1)
    for bad in ([np.nan, 1.0], [-np.inf, -np.inf], [np.inf, 0.0]):
        assert OF.sample(bad, 0.5)[0] == -1 and OF.sample(bad, 0.5)[2] == 0
    assert OF.sample([0.0, 1.0], 0.5, temperature=-1.0)[0] == -1 and OF.sample([0.0, 1.0], 0.5, top_p=np.nan)[0] == -1
    out, n = OF.masked(X, top_k=2)
    assert n == 2 and out[1] == X[1] and out[3] == X[3] and np.isneginf(out[[0, 2, 4]]).all()


def test_shares_of_many_draws():
    rng = np.random.default_rng(0)
    got = np.bincount([OF.sample(X, u, top_p=0.86)[0] for u in rng.random(4000)], minlength=5) / 4000
    assert np.abs(got - [0, 0.4, 0.2, 0.4, 0]).max() < 0.04 and got[0] == got[4] == 0

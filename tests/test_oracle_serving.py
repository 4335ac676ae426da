"""Pins of the oracles of the serving operators: small cases by hand, and what follows from the definitions."""
import numpy as np
import pytest

from oracle import kv4 as OK
from oracle import page_tables as OP
from oracle import sampled_acceptance as OA


def test_page_tables_by_hand():
    table = [[7, -1, -1], [-1, -1, -1], [3, 4, -1]]
    got = OP.page_tables([18, 16, 40], [3, 16, 2], [1, 0, 2], [20, 21, 22], table, 24)
    assert table == [[7, 20, -1], [21, -1, -1], [3, 4, 22]]
    assert got[0] == [2, 1, 3] and got[1] == [0, 3, 19, 21] and got[3] == [21, 3, 0]
    assert got[2] == [7 * 16 + 15, 20 * 16, 20 * 16 + 1] + [21 * 16 + i for i in range(16)] + [22 * 16 + 6, 22 * 16 + 7] + [-1] * 3


def test_page_tables_refuse_in_order():
    # the second asks for two pages of one that is left; the third needs none and is served, the fourth cannot be any more
    table = [[-1] * 3 for _ in range(4)]
    table[2][0] = 9
    got = OP.page_tables([16, 20, 16, 1], [1, 1, 1, 1], [0, 0, 1, 0], [5, 6], table, 4)
    assert table == [[5, -1, -1], [-1] * 3, [9, -1, -1], [-1] * 3]
    assert got[0] == [1, 0, 1, 0] and got[2] == [5 * 16 + 15, -1, 9 * 16 + 15, -1] and got[3] == [4, 3, 2]


def test_numbers_are_the_nearest():
    rng = np.random.default_rng(0)
    x = OK.bf16(rng.normal(size=(40, 2, 128)).astype(np.float32))
    n, scale, low = OK.quantise(x)
    g = x.reshape(40, 2, 2, 64).astype(np.float64)
    off = np.abs(OK.values(n, scale, low).reshape(g.shape) - g)
    for other in range(16):
        assert (off <= np.abs(low[..., None] + scale[..., None] * other - g) + 1e-12).all()
    assert (low == g.min(-1)).all() and (n.min(-1) == 0).all() and (n.max(-1) == 15).all()
    # half a step, and what the scale's rounding takes from the largest
    assert (off <= scale[..., None] * (0.5 + 15 * 2.0 ** -8)).all()


def test_numbers_at_borders():
    x = np.zeros(32, dtype=np.float32)
    x[:6] = [0, 15, 0.5, 1.5, 2.5, 2.4999998]                # scale 1: ties go to the even number
    n, scale, low = OK.quantise(x)
    assert scale[0] == 1 and low[0] == 0 and n[0, :6].tolist() == [0, 15, 0, 2, 2, 2]
    n, scale, low = OK.quantise(np.full(64, -3.25, dtype=np.float32))
    assert scale[0] == 0 and (n == 0).all() and (OK.values(n, scale, low) == -3.25).all()
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones(128, dtype=np.float32)
        x[70] = bad
        v = OK.values(*OK.quantise(x))
        assert (v[:64] == 1).all() and np.isnan(v[64:]).all()


def test_attention_against_a_plain_softmax():
    rng = np.random.default_rng(1)
    k, v = (OK.quantise(rng.normal(size=(21, 2, 32)).astype(np.float32)) for _ in range(2))
    q = rng.normal(size=(3, 4, 32))
    out, bound = OK.attention(q, k, v, 3, 0.2)
    for i in range(3):
        for h in range(4):
            x = 0.2 * OK.values(*k)[:19 + i, h // 2] @ q[i, h]
            p = np.exp(x) / np.exp(x).sum()
            assert np.allclose(out[i, h], p @ OK.values(*v)[:19 + i, h // 2], atol=1e-12)
    assert (bound > 0).all() and bound.max() < 0.05
    assert (OK.attention(q, tuple(t[:1] for t in k), tuple(t[:1] for t in v), 3, 0.2)[0][:2] == 0).all()   # two rows before the only token


def test_draws_follow_the_target():
    """Drafts drawn from q and verified against p: what is emitted first is distributed as p, with q given and with fixed drafts."""
    rng = np.random.default_rng(2)
    logits = rng.normal(size=(2, 6)) * 1.5
    p = OA.distribution(logits[0], 0.7)
    q = rng.dirichlet(np.ones(6))
    n = 40000
    for probs in (q[None], None):
        seen = np.zeros(6)
        for _ in range(n):
            d = rng.choice(6, p=q) if probs is not None else 3
            seen[OA.accept(logits, [d], probs, 0.7, rng.random((2, 2)))[1][0]] += 1
        assert np.abs(seen / n - p).max() < 5 * np.sqrt(0.25 / n)      # five standard deviations of a share


@pytest.mark.parametrize("u, want", [(0.0, 1), (0.2499, 1), (0.25, 3), (0.9999, 3)])
def test_draw_takes_the_lowest_token_past_the_sum(u, want):
    assert OA.draw(np.array([0.0, 1.0, 0.0, 3.0, 0.0]), u) == want


def test_rows_without_a_distribution():
    ok = [0.0, 1.0]
    for bad in ([np.nan, 0.0], [np.inf, 0.0], [-np.inf, -np.inf]):
        m, tokens, logp = OA.accept([ok, bad, ok], [1, 0], None, 0.0, np.zeros((3, 2)))
        assert (m, tokens) == (1, [1, -1]) and np.isnan(logp[1])
    assert OA.distribution(ok, -1.0) is None and OA.distribution(ok, float("nan")) is None
    assert OA.accept([ok, ok], [0], None, 0.0, np.zeros((2, 2)))[:2] == (0, [1])     # greedy: another token than the largest

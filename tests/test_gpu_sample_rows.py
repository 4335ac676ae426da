"""tasc_sample and tasc_filter_logits over rows as masks and vocabularies make them, against their oracle in 64 bits (tokens and counts equal, probabilities within the
tolerance that test_gpu_sample derives)."""
import itertools

import numpy as np
import pytest

from test_gpu_sample import check

pytestmark = pytest.mark.gpu
f32 = lambda *v: np.array(v, dtype=np.float32)


def type_of(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("live", ["uniform", "normal"])
@pytest.mark.parametrize("mask", [-5e3, -1e4, -1e9])
@pytest.mark.parametrize("vocab", [50257, 151936])
def test_top_p_and_min_p_beside_a_finite_mask(vocab, mask, live, dtype):
    """Masks that are large numbers instead of -infinity stretch the span of a flat row over many temperatures; top-p keeps less than min-p in some rows, more in others"""
    rng = np.random.default_rng(vocab + int(-mask) % 1000 + len(live))
    t, p, m = f32(*itertools.product((0.6, 1.0, 1.2), (0.8, 0.9, 0.95), (0.01, 0.05, 0.1))).T.copy()
    x = rng.uniform(0, 10, (len(t), vocab)) if live == "uniform" else rng.standard_normal((len(t), vocab))
    x[:, ::97] = mask
    check(x, rng.random(len(t)).astype(np.float32), t=t, p=p, m=m, dtype=type_of(dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_top_k_and_min_p_over_few_logits(dtype):
    """2^24 tokens of three logits, more of each in a part of the row than 16 bits count: top-k cuts the first logit's tokens, where min-p alone keeps all of them, or the second's"""
    rng = np.random.default_rng(12)
    x = rng.integers(0, 3, (2, 1 << 24)) * -0.5
    check(x, f32(0.4, 0.9), k=np.array([5000000, 8000000], dtype=np.int32), m=f32(0.74, 0.5), dtype=type_of(dtype))


@pytest.mark.parametrize("vocab", [900, 30000])
def test_words_of_a_row_over_those_that_it_reads(vocab):
    """token, logprob and kept in the place of parameters and random numbers: as beside them"""
    import torch
    import paper_2602_24174_amd as T
    from test_gpu_sample import dev, logits_of, settings
    rng = np.random.default_rng(vocab)
    rows = 64
    x, u = dev(logits_of(rng, rows, vocab, "flat").astype(np.float32)), dev(rng.random(rows).astype(np.float32))
    x[::2, :8] += 9.0                                      # every other row keeps few tokens
    per = [dev(a) for a in settings(rng, rows)]
    new = lambda t: torch.zeros(rows, dtype=t, device="cuda")
    want = new(torch.int32), new(torch.float32), new(torch.int32)
    T.tasc_sample(x, u, want[0], *per, want[1], want[2])
    masks, counts = torch.zeros((rows, 1, vocab), device="cuda"), torch.zeros((rows, 1), dtype=torch.int32, device="cuda")
    T.tasc_filter_logits(x[:, None], masks, *per, counts)
    for i, name in enumerate(("u", "t", "k", "p", "m")):
        at = dict(zip(("u", "t", "k", "p", "m"), (u.clone(), *(a.clone() for a in per))))
        for out in range(3):
            args = {n: a.clone() for n, a in at.items()}
            got = [torch.zeros_like(w) for w in want]
            got[out] = args[name].view(got[out].dtype)
            T.tasc_sample(x, args["u"], got[0], args["t"], args["k"], args["p"], args["m"], got[1], got[2])
            assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in zip(got, want)), (name, out)
        if name != "u":
            args = {n: a.clone() for n, a in at.items()}
            out, kept = torch.zeros_like(masks), args[name].view(torch.int32)[:, None]
            T.tasc_filter_logits(x[:, None], out, args["t"], args["k"], args["p"], args["m"], kept)
            assert torch.equal(out, masks) and torch.equal(kept, counts), name


def by_index(rng, rows, vocab, kind):
    """Logits whose level or mask goes by the token's index, as a vocabulary's do"""
    x = rng.standard_normal((rows, vocab)) * 1.5
    v = np.arange(vocab)
    if kind.startswith("falling"):
        x -= float(kind[7:]) * np.log10(1 + v)
    elif kind.startswith("below"):                          # live below an index, and one token that ends a text
        x[:, (v >= int(kind[5:]) * vocab // 151936) & (v != vocab * 9 // 10)] = -np.inf
    elif kind == "last":                                    # nothing in the parts' first loads
        x[:, :vocab - vocab // 20] = -np.inf
    elif kind == "blocks":
        x[:, v // 3000 % 2 == 0] = -np.inf
    return x


@pytest.mark.parametrize("rows, vocab, dtype", [(1, 151936, "f32"), (24, 151936, "f32"), (64, 151936, "f32"), (24, 151936, "bf16"), (24, 50257, "f32"), (64, 5003, "f32")])
@pytest.mark.parametrize("kind", ["falling0.5", "falling1", "below20000", "below32000", "below100000", "last", "blocks"])
def test_logits_that_go_by_the_index(kind, rows, vocab, dtype):
    rng = np.random.default_rng(rows + vocab + len(kind))
    x = by_index(rng, rows, vocab, kind)
    i = np.arange(rows)
    # a row each without filters, by top-p, by top-k, by both, by all three, by min-p
    k = np.where(np.isin(i % 6, (2, 3, 4)), rng.choice((5, 40, 100, 1000), rows), 0).astype(np.int32)
    p = np.where(np.isin(i % 6, (1, 3, 4)), rng.uniform(0.5, 0.98, rows), 1.0).astype(np.float32)
    m = np.where(np.isin(i % 6, (4, 5)), rng.uniform(0.001, 0.1, rows), 0.0).astype(np.float32)
    if rows == 1:
        k[:], p[:] = 100, 0.9
    check(x, rng.random(rows).astype(np.float32), t=rng.uniform(0.5, 1.5, rows).astype(np.float32), k=k, p=p, m=m, dtype=type_of(dtype), mask=rows < 64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1279, 1280, 1281, 1282])
@pytest.mark.parametrize("kind", ["peaked", "flat", "masked", "ties", "equal", "wide", "zeros"])
def test_the_longest_rows_that_are_their_own_lists(kind, vocab, dtype):
    from test_gpu_sample import logits_of, settings
    rng = np.random.default_rng(vocab + len(kind))
    check(logits_of(rng, 16, vocab, kind), rng.random(16).astype(np.float32), *settings(rng, 16), dtype=type_of(dtype))

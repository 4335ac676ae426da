"""Attention over values up to the largest that the cache holds: results as finite as the values are, held to the oracle's bound."""
import numpy as np
import pytest

from oracle import kv4 as OK
from test_gpu_kv4 import Batch

pytestmark = pytest.mark.gpu


def give_values(batch, b, v):
    """Puts other values (float32 [tokens, heads, head_dim]) beside a sequence's keys."""
    import torch
    import paper_2602_24174_amd as T
    pos = np.arange(len(v))
    table = batch.table[b].cpu().numpy()
    slots = torch.tensor(table[pos // 16] * 16 + pos % 16, dtype=torch.int32, device="cuda")
    k, old = (torch.zeros(v.shape, device="cuda") for _ in range(2))
    T.tasc_kv4_read(batch.cache, slots, k, old)
    new = torch.tensor(v).cuda()
    T.tasc_kv4_append(batch.cache, k, new, slots)
    batch.k[b], batch.v[b] = OK.quantise(k.cpu().numpy()), OK.quantise(v)
    return slots


def large(rng, n, heads, hd):
    """Every kind of group among ordinary ones: no range, a narrow one, all of fp32's range, half of it above or below zero."""
    x = rng.normal(size=(n, heads, hd)).astype(np.float32)
    wide = rng.uniform(-1, 1, size=x.shape)
    kinds = [lambda w: w * 0 + 3.2e38, lambda w: w * 0 - 3.2e38, lambda w: 1.6e38 * w, lambda w: 1.6e38 * (w + 1), lambda w: -1e38 * (w + 2), lambda w: w * 0 + 1e36,
             lambda w: 3e38 + 1e33 * w, lambda w: 1e30 * w]
    for at, t in enumerate(range(1, n, 3)):
        x[t] = kinds[at % len(kinds)](wide[t]).astype(np.float32)
    return x


# one tile; eight waves that share a sequence's tiles; two, with key chunks joined by either merge; waves with rows of their own
@pytest.mark.parametrize("lens, rows, heads, kv_heads", [([20, 33], [16, 2], 4, 2), ([700, 90], [1, 1], 6, 2), ([2050], [9], 12, 2), ([2050], [1], 12, 2), ([9000], [1], 4, 1),
                                                         ([150, 200] * 22, [150, 129] * 22, 12, 2)])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_values_of_every_size(hd, lens, rows, heads, kv_heads):
    print(f"{heads}/{kv_heads} x {hd}: {len(lens)} sequences, tokens {lens[:2]}, rows {rows[:2]}", flush=True)
    batch = Batch(lens, rows, heads, kv_heads, hd, seed=hd)
    rng = np.random.default_rng(hd)
    some = range(min(len(lens), 2))
    for b in some:
        give_values(batch, b, large(rng, lens[b], kv_heads, hd))
    got = batch.run().float().cpu().numpy()
    q = batch.q.float().cpu().numpy().astype(np.float64)
    for b in some:
        n = rows[b]
        at = slice(batch.off[b], batch.off[b + 1])
        want, bound = OK.attention(q[at], batch.k[b], batch.v[b], n, batch.scale)
        assert np.isfinite(want).all()
        assert (np.abs(got[at] - want) <= bound).all(), (b, int((~np.isfinite(got[at])).sum()), float(np.nanmax(np.abs(got[at] - want) / bound)))


def test_rows_before_a_large_value():
    """Rows that do not see the large token are, bit for bit, what they are without it."""
    for hd in (64, 128):
        batch = Batch([45, 300], [6, 3], 4, 2, hd)
        rng = np.random.default_rng(hd)
        ordinary = [rng.normal(size=(n, 2, hd)).astype(np.float32) for n in batch.lens]
        for b, v in enumerate(ordinary):
            give_values(batch, b, v)
        clean = batch.run()
        for b, v in enumerate(ordinary):
            v[-1] = 3e38
            give_values(batch, b, v)
        out = batch.run()
        seen = [5, 8]                                         # the last rows
        assert all((out[r] == clean[r]).all() for r in range(9) if r not in seen)
        assert all(((out[r].float() > 1e30) & (out[r].float() < 3.4e38)).all() for r in seen)

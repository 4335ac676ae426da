"""Every kernel of the attention over the 4-bit cache, at the calls of kv4_shapes.py: results against the oracle, and what only shows where a
kernel does its own masking and joining.  A kernel is checked on a few of a call's sequences, bit for bit against itself on all."""
import numpy as np
import pytest

from kv4_shapes import FOUR, ROWS, TWO
from oracle import kv4 as OK
from test_gpu_kv4 import Batch

pytestmark = pytest.mark.gpu

CALLS = {f"{kind}-{name}": call for kind, cases in (("rows", ROWS), ("four", FOUR), ("two", TWO)) for name, (call, _) in cases.items()}
# a call of every kernel
EACH = ["rows-hd32", "rows-hd64", "rows-hd128", "four-hd32", "four-hd64", "four-hd128", "four-chunks", "two-many_heads", "two-split"]


def batch_of(name, seed=1, q_scale=1.0):
    """Ragged lengths and rows up to the call's bounds, the first sequence at both of them."""
    B, kvh, heads, hd, rows, kv = CALLS[name]
    rng = np.random.default_rng(seed)
    n = rng.integers(1 if rows == 1 else 0, rows + 1, B)
    n[0] = rows
    lens = np.maximum(rng.integers(max(1, kv // 3), kv + 1, B), n)
    lens[0] = kv
    if B > 3:
        n[3] = rows                                           # a whole prompt, or a row that sees itself alone
        lens[3] = rows
    print(f"{name}: {B} sequences, {heads}/{kvh} x {hd}, {n.sum()} rows", flush=True)
    b = Batch(lens.tolist(), n.tolist(), heads, kvh, hd, seed=seed, q_scale=q_scale)
    b.bounds = dict(max_rows=rows, max_kv=kv)
    return b


def some_of(batch):
    return sorted({0, 1 % len(batch.n), 3 % len(batch.n), len(batch.n) - 1})


def check_some(batch, out):
    got, q = out.float().cpu().numpy(), batch.q.float().cpu().numpy()
    assert (got[batch.off[-1]:] == 7).all()
    for b in some_of(batch):
        rows = slice(batch.off[b], batch.off[b + 1])
        want, bound = OK.attention(q[rows].astype(np.float64), batch.k[b], batch.v[b], batch.n[b], batch.scale)
        assert (np.abs(got[rows] - want) <= bound).all(), b


@pytest.mark.parametrize("name", list(CALLS))
def test_against_the_oracle(name):
    batch = batch_of(name)
    out = batch.run(**batch.bounds)
    check_some(batch, out)
    assert out[:batch.off[-1]].isfinite().all()


@pytest.mark.parametrize("name", EACH)
def test_rows_are_independent_and_calls_repeat(name):
    import torch
    batch = batch_of(name)
    first = batch.run(**batch.bounds)
    assert torch.equal(first, batch.run(**batch.bounds))
    q = batch.q.clone()
    q[1::2] = 3.0
    assert torch.equal(batch.run(q=q, **batch.bounds)[:batch.off[-1]:2], first[:batch.off[-1]:2])


@pytest.mark.parametrize("name", EACH)
def test_pages_outside_the_pool(name):
    """In every third sequence two pages are none: their tokens are not seen."""
    import torch
    batch = batch_of(name, seed=2)
    table = batch.table.clone()
    gone = (1, 3)
    table[::3, gone[0]], table[::3, gone[1]] = -1, batch.cache.n_pages
    table[::6, gone[0]], table[::6, gone[1]] = -2147483648, 2147483647
    out, clean = batch.run(table=table, **batch.bounds), batch.run(**batch.bounds)
    q = batch.q.float().cpu().numpy().astype(np.float64)
    for b in some_of(batch):
        n, rows = batch.lens[b], batch.n[b]
        at = slice(batch.off[b], batch.off[b + 1])
        if b % 3:
            assert torch.equal(out[at], clean[at])
            continue
        keep = np.array([t for t in range(n) if t // 16 not in gone])
        for i in {0, rows // 2, rows - 1} if rows else ():
            seen = keep[keep <= n - rows + i]
            want, bound = OK.attention(q[batch.off[b] + i][None], tuple(t[seen] for t in batch.k[b]), tuple(t[seen] for t in batch.v[b]), 1, batch.scale)
            assert (np.abs(out[batch.off[b] + i].float().cpu().numpy() - want[0]) <= bound[0]).all(), (b, i)
    assert (batch.run(table=torch.full_like(table, -1), **batch.bounds)[:batch.off[-1]] == 0).all()


@pytest.mark.parametrize("name", EACH)
def test_numbers_that_are_none_where_they_are_masked(name):
    """A sequence's last token of infinities and NaN: its last row alone sees it; queries of NaN spoil their own row alone."""
    import torch
    import paper_2602_24174_amd as T
    batch = batch_of(name, seed=3)
    clean = batch.run(**batch.bounds)
    hd, kvh = batch.cache.head_dim, batch.cache.n_kv_heads
    some = [b for b in some_of(batch) if batch.n[b] > 0]
    bad = torch.full((len(some), kvh, hd), float("inf"), device="cuda")
    bad[:, 0, 3] = float("nan")
    last = [batch.lens[b] - 1 for b in some]
    slots = torch.tensor([int(batch.table[b, t // 16]) * 16 + t % 16 for b, t in zip(some, last)], dtype=torch.int32, device="cuda")
    T.tasc_kv4_append(batch.cache, bad, bad, slots)
    spoilt = {int(batch.off[b + 1]) - 1 for b in some}
    batch.q[int(batch.off[-1]):] = float("inf")
    if batch.n[0] > 2:
        batch.q[1] = float("nan")
        spoilt.add(1)
    out = batch.run(**batch.bounds)
    whole = torch.tensor([r for r in range(int(batch.off[-1])) if r not in spoilt], device="cuda")
    assert torch.equal(out[whole], clean[whole]) and all(out[r].isnan().all() for r in spoilt)
    assert (out[int(batch.off[-1]):] == 7).all()


@pytest.mark.parametrize("name", EACH)
def test_bounds_offsets_and_lengths(name):
    """Rows beyond max_rows stay as they were; offsets and lengths that make no sense."""
    import torch
    batch = batch_of(name, seed=4)
    clean = batch.run(**batch.bounds)
    # a sequence that claims the next one's rows, too: its first max_rows rows, as the last ones but those of that many
    most = batch.bounds["max_rows"]
    off = batch.row_off.clone()
    nothing = torch.full_like(clean, 7.0)
    batch.row_off = torch.tensor([-2147483648, 5, 2, 2147483647] + [-3] * (len(batch.n) - 3), dtype=torch.int32, device="cuda")[:len(batch.n) + 1]
    out = batch.run(**batch.bounds)
    if len(batch.n) > 2:                                      # the third sequence has rows 2 .. of very many, which see nothing
        assert (out[2:min(2 + most, len(out))] == 0).all() and torch.equal(out[:2], nothing[:2]) and torch.equal(out[2 + most:], nothing[2 + most:])
    batch.row_off, kv = off, batch.kv_len
    batch.kv_len = kv.clone()
    batch.kv_len[1::2] = -1
    batch.kv_len[1::4] = -2147483648
    out = batch.run(**batch.bounds)
    for b in some_of(batch):
        at = slice(batch.off[b], batch.off[b + 1])
        assert (out[at] == 0).all() if b % 2 else torch.equal(out[at], clean[at])


@pytest.mark.parametrize("name", ["rows-hd128", "rows-least_pairs", "two-split"])
def test_rows_beyond_the_bound(name):
    batch = batch_of(name, seed=5)
    most = batch.bounds["max_rows"]
    wide = Batch([most + 60, 40, most + 9] + batch.lens[3:], [most + 40, 3, most + 1] + batch.n[3:], batch.heads, batch.cache.n_kv_heads, batch.cache.head_dim, seed=6)
    out = wide.run(max_rows=most, max_kv=batch.bounds["max_kv"]).float().cpu().numpy()
    q = wide.q.float().cpu().numpy().astype(np.float64)
    for b in range(min(3, len(wide.n))):
        first, n, kept = wide.off[b], wide.n[b], min(wide.n[b], most)
        want, bound = OK.attention(q[first:first + n], wide.k[b], wide.v[b], n, wide.scale)
        assert (np.abs(out[first:first + kept] - want[:kept]) <= bound[:kept]).all() and (out[first + kept:first + n] == 7).all()


@pytest.mark.parametrize("name", EACH)
def test_strided_rows_and_untouched_elements(name):
    import torch
    batch = batch_of(name, seed=7)
    want = batch.run(**batch.bounds)
    rows, heads, hd = batch.q.shape
    wide = torch.randn((rows, heads + 4, hd), device="cuda").bfloat16()
    wide[:, 2:2 + heads] = batch.q
    out = torch.full((rows, heads + 3, hd), 5.0, dtype=torch.bfloat16, device="cuda")
    batch.run(q=wide[:, 2:2 + heads], out=out[:, 1:1 + heads], **batch.bounds)
    end = int(batch.off[-1])
    assert torch.equal(out[:end, 1:1 + heads], want[:end]) and (out[:, 0] == 5).all() and (out[:, 1 + heads:] == 5).all() and (out[end:] == 5).all()


@pytest.mark.parametrize("name", EACH)
def test_large_scores(name):
    batch = batch_of(name, seed=8, q_scale=30.0)
    check_some(batch, batch.run(**batch.bounds))

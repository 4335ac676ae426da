"""The 4-bit cache and the attention over it against float64.

Values read back are the oracle's numbers rounded to the output's type once (and once in between, for bf16: low + scale c in fp32
first).  Attention is held to the bound that oracle/kv4.py derives element by element."""
import numpy as np
import pytest

from oracle import kv4 as OK

pytestmark = pytest.mark.gpu

HEADS = [(1, 32), (3, 32), (2, 64), (3, 64), (1, 128), (5, 128)]


def tokens(rng, rows, heads, hd, dtype):
    import torch
    x = rng.normal(size=(rows, heads, hd)).astype(np.float32)
    x[..., 3::29] *= 6
    return torch.tensor(x).to(getattr(torch, dtype)).cuda()


def dirty_cache(pages, heads, hd):
    """A pool in which every byte is set: what nothing has written reads as NaN."""
    import paper_2602_24174_amd as T
    c = T.Kv4Cache(pages, heads, hd)
    c.pool.fill_(0xFF)
    return c


def read(cache, slots, dtype="float32"):
    import torch
    import paper_2602_24174_amd as T
    out = [torch.full((len(slots), cache.n_kv_heads, cache.head_dim), 99, dtype=getattr(torch, dtype), device="cuda") for _ in range(2)]
    T.tasc_kv4_read(cache, slots, *out)
    return [o.float().cpu().numpy() for o in out]


def held(x):
    """What the cache holds of x, in the float32 that low + scale c is computed in."""
    return OK.values(*OK.quantise(x.float().cpu().numpy())).astype(np.float32)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("heads, hd", HEADS)
def test_round_trip(heads, hd, dtype):
    import torch
    import paper_2602_24174_amd as T
    rng = np.random.default_rng(hd + heads)
    for rows in (1, 17, 130):
        print(f"{rows} rows of {heads} x {hd} {dtype}", flush=True)
        pages = rows // 16 + 3
        cache = dirty_cache(pages, heads, hd)
        before = cache.pool.clone()
        slots = torch.tensor(rng.permutation(pages * 16)[:rows], dtype=torch.int32, device="cuda")
        slots[rows // 2::5] = -1
        if rows > 3:
            slots[2], slots[3] = pages * 16, 2147483647       # outside the pool
        k, v = tokens(rng, rows, heads, hd, dtype), tokens(rng, rows, heads, hd, dtype)
        T.tasc_kv4_append(cache, k, v, slots)
        inside = ((slots >= 0) & (slots < pages * 16)).cpu().numpy()
        for got, x in zip(read(cache, slots), (k, v)):
            assert (got[inside] == held(x)[inside]).all() and (got[~inside] == 0).all()
        for got, x in zip(read(cache, slots, "bfloat16"), (k, v)):
            assert (got[inside] == OK.bf16(held(x))[inside]).all()
        # nothing but the named slots: their bytes back to what they were, and the pool is
        other = torch.tensor(np.setdiff1d(np.arange(pages * 16), slots.cpu().numpy()), dtype=torch.int32, device="cuda")
        assert all(np.isnan(x).all() for x in read(cache, other))
        assert (cache.pool != before).any() == inside.any()


def test_strides_and_alignment():
    """Keys and values inside the rows of a fused projection; rows that start at any element; one row for all (stride 0)."""
    import torch
    import paper_2602_24174_amd as T
    rng = np.random.default_rng(3)
    for dtype in ("float32", "bfloat16"):
        for pad in (0, 1, 3, 8):
            qkv = tokens(rng, 20, 9, 64, dtype).reshape(20, -1)
            wide = torch.cat([torch.zeros((20, pad), dtype=qkv.dtype, device="cuda"), qkv], 1)
            k, v = (wide.as_strided((20, 2, 64), (wide.stride(0), 64, 1), pad + at * 64) for at in (5, 7))
            cache, slots = dirty_cache(2, 2, 64), torch.arange(20, dtype=torch.int32, device="cuda") + 5
            T.tasc_kv4_append(cache, k, v, slots)
            for got, x in zip(read(cache, slots), (k, v)):
                assert (got == held(x)).all()
        one = tokens(rng, 1, 2, 64, dtype).expand(20, 2, 64)
        T.tasc_kv4_append(cache, one, one, slots)
        assert (read(cache, slots)[1] == held(one)).all()


def test_groups_that_are_no_numbers():
    import torch
    import paper_2602_24174_amd as T
    for hd in (32, 64, 128):
        x = torch.ones((6, 1, hd), device="cuda")
        x[:, 0, 1] = 2
        x[0, 0, 5], x[1, 0, 5], x[2, 0, 5] = float("nan"), float("inf"), float("-inf")
        x[3, 0, 4], x[3, 0, 5] = 3e38, -3e38                  # a range beyond fp32
        x[4] = 1e-42                                          # subnormal, no range
        x[5, 0, 5] = 1 + 2e-39
        cache, slots = dirty_cache(1, 1, hd), torch.arange(6, dtype=torch.int32, device="cuda")
        T.tasc_kv4_append(cache, x, x, slots)
        for got in read(cache, slots):
            assert np.array_equal(got, held(x), equal_nan=True)
            assert np.isnan(got[:4, 0, :min(hd, 64)]).all() and np.isfinite(got[:, 0, 64:]).all() and np.isfinite(got[4:]).all()


# ------------------------------------------------------------------------------------------------ attention
class Batch:
    """Sequences of given lengths and rows in a pool of shuffled pages whose unwritten bytes are all set."""

    def __init__(self, lens, rows, heads, kv_heads, hd, seed=0, extra_pages=2, q_scale=1.0):
        import torch
        import paper_2602_24174_amd as T
        self.lens, self.n, self.heads = list(lens), list(rows), heads
        rng = np.random.default_rng(seed)
        need = [-(-max(n, 1) // 16) for n in lens]
        cols, pages = max(need) + 1, sum(need) + extra_pages
        order = rng.permutation(pages)
        table = np.full((len(lens), cols), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.cache = dirty_cache(pages, kv_heads, hd)
        self.k, self.v = [], []
        for b, n in enumerate(lens):
            k, v = tokens(rng, n, kv_heads, hd, "bfloat16"), tokens(rng, n, kv_heads, hd, "bfloat16")
            pos = np.arange(n)
            slots = torch.tensor(table[b, pos // 16] * 16 + pos % 16, dtype=torch.int32, device="cuda")
            T.tasc_kv4_append(self.cache, k, v, slots)
            self.k.append(OK.quantise(k.float().cpu().numpy()))
            self.v.append(OK.quantise(v.float().cpu().numpy()))
        off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.off, self.table = off, torch.tensor(table, device="cuda")
        self.row_off, self.kv_len = torch.tensor(off, device="cuda"), torch.tensor(np.asarray(lens, dtype=np.int32), device="cuda")
        self.q = torch.tensor(rng.normal(size=(off[-1] + 3, heads, hd)).astype(np.float32) * q_scale).bfloat16().cuda()
        self.scale = hd ** -0.5

    def run(self, q=None, out=None, max_rows=None, max_kv=None, workspace=None, table=None):
        import torch
        import paper_2602_24174_amd as T
        q = self.q if q is None else q
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
        T.tasc_kv4_attention(self.cache, q, self.table if table is None else table, self.row_off, self.kv_len, max_rows or max(self.n), max_kv or max(self.lens), self.scale, out,
                             workspace)
        return out

    def check(self, out):
        got = out.float().cpu().numpy()
        q = self.q.float().cpu().numpy()
        assert (got[self.off[-1]:] == 7).all(), "rows behind the last sequence"
        for b, n in enumerate(self.n):
            rows = slice(self.off[b], self.off[b + 1])
            want, bound = OK.attention(q[rows].astype(np.float64), self.k[b], self.v[b], n, self.scale)
            off = np.abs(got[rows] - want)
            assert (off <= bound).all(), (b, float((off / np.maximum(bound, 1e-30)).max()))


@pytest.mark.parametrize("heads, kv_heads, hd", [(1, 1, 32), (9, 3, 64), (14, 2, 64), (12, 2, 128), (8, 8, 128), (6, 3, 32)])
def test_attention_lengths(heads, kv_heads, hd):
    """One token to several tiles, pages and tiles that end inside, one row to more than a tile of pairs, sequences without rows."""
    for lens, rows in (([1], [1]), ([15, 16, 17, 31, 32, 33, 1, 64], [1] * 8), ([40, 5, 130, 97], [3, 5, 9, 0]), ([70, 300], [17, 40])):
        print(f"{heads}/{kv_heads} x {hd}: tokens {lens}, rows {rows}", flush=True)
        batch = Batch(lens, rows, heads, kv_heads, hd, seed=sum(lens))
        batch.check(batch.run())


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_attention_split_over_keys(hd):
    """Few sequences of many tokens: the keys are cut into chunks that are joined; a short one among them leaves chunks empty."""
    for lens, rows, heads, kv_heads in (([5000], [1], 4, 1), ([3001, 40, 1], [2, 2, 1], 4, 2), ([2050, 2048], [9, 1], 12, 2)):
        print(f"tokens {lens}, rows {rows}", flush=True)
        batch = Batch(lens, rows, heads, kv_heads, hd, seed=sum(lens))
        batch.check(batch.run())


@pytest.mark.parametrize("heads, kv_heads, hd", [(12, 2, 128), (14, 2, 64), (4, 4, 32)])
def test_attention_prompts(heads, kv_heads, hd):
    """Whole prompts (no cached token before them) and chunks of them, with enough sequences that waves have rows of their own."""
    for lens, rows in (([150, 200, 90, 260] * 8, [150, 70, 90, 256] * 8), ([300] * 40, [129] * 40)):
        print(f"{len(lens)} prompts, {sum(rows)} rows", flush=True)
        batch = Batch(lens, rows, heads, kv_heads, hd, seed=len(lens))
        batch.check(batch.run())


def test_rows_that_see_nothing():
    """More rows than tokens: the first ones stand before the first key."""
    for hd in (32, 128):
        batch = Batch([3, 0, 20], [5, 2, 30], 4, 2, hd)
        out = batch.run()
        batch.check(out)
        assert (out[:2] == 0).all() and (out[5:7] == 0).all() and (out[7:17] == 0).all()


def test_rows_beyond_the_bound_are_left_out():
    """max_rows below a sequence's rows: its first ones are as they are without the bound, the others stay as they were."""
    import torch
    for lens, rows, most, heads in (([40, 9], [7, 3], 4, 4), ([300], [200], 70, 12), ([5, 64], [9, 2], 3, 4)):
        batch = Batch(lens, rows, heads, 2, 64)
        all_of, some = batch.run().float().cpu().numpy(), batch.run(max_rows=most).float().cpu().numpy()
        q = batch.q.float().cpu().numpy().astype(np.float64)
        for b, n in enumerate(rows):
            first, kept = batch.off[b], min(n, most)
            want, bound = OK.attention(q[first:first + n], batch.k[b], batch.v[b], n, batch.scale)
            assert (np.abs(some[first:first + kept] - want[:kept]) <= bound[:kept]).all() and (np.abs(all_of[first:first + n] - want) <= bound).all()
            assert (some[first + kept:first + n] == 7).all()


def test_lengths_and_rows_that_make_no_sense():
    """Negative lengths: rows that see nothing.  Offsets that fall or begin below 0: no rows.  Offsets beyond the rows: those that exist."""
    import torch
    batch = Batch([40, 40, 40, 40], [2, 3, 2, 2], 4, 2, 64)
    clean = batch.run()
    one = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    batch.kv_len = one([40, -2147483648, -1, 40])
    out = batch.run()
    assert torch.equal(out[:2], clean[:2]) and (out[2:7] == 0).all() and torch.equal(out[7:], clean[7:])
    batch.kv_len, batch.row_off = one([40] * 4), one([-2147483648, 5, 2, 2147483647, -3])
    out = batch.run(max_rows=3)
    assert (out[:2] == 7).all() and (out[5:] == 7).all()        # the third sequence has rows 2, 3, 4 of very many, which see nothing
    assert (out[2:5] == 0).all()


def test_pages_outside_the_pool():
    """Their tokens are not seen, and nothing is read there."""
    import torch
    batch = Batch([100, 64], [2, 1], 4, 2, 64)
    table = batch.table.clone()
    table[0, 1], table[0, 4], table[1, 0], table[1, 3] = -1, batch.cache.n_pages, -2147483648, 2147483647
    out = batch.run(table=table)
    q = batch.q.float().cpu().numpy().astype(np.float64)
    for b, gone in enumerate(([1, 4], [0, 3])):
        n, rows = batch.lens[b], batch.n[b]
        keep = np.array([t for t in range(n) if t // 16 not in gone])
        for i in range(rows):
            seen = keep[keep <= n - rows + i]
            want, bound = OK.attention(q[batch.off[b] + i][None], tuple(t[seen] for t in batch.k[b]), tuple(t[seen] for t in batch.v[b]), 1, batch.scale)
            assert (np.abs(out[batch.off[b] + i].float().cpu().numpy() - want[0]) <= bound[0]).all()
    assert (batch.run(table=torch.full_like(table, -1))[:3] == 0).all()


def test_numbers_that_are_none_where_they_are_masked():
    """NaN and infinity in tokens behind a row's last one, in later rows' queries, and in rows that no sequence has."""
    import torch
    import paper_2602_24174_amd as T
    for hd in (64, 128):
        batch = Batch([45, 80], [4, 1], 4, 2, hd)
        clean = batch.run()
        bad = torch.full((1, 2, hd), float("inf"), device="cuda")
        bad[0, 0, 3] = float("nan")
        slot = batch.table[0, 2:3] * 16 + 44 % 16               # the last token of the first sequence: rows 0 .. 2 do not see it
        T.tasc_kv4_append(batch.cache, bad, bad, slot)
        batch.q[3], batch.q[5:] = float("nan"), float("inf")
        out = batch.run()
        assert torch.equal(out[:3], clean[:3]) and torch.equal(out[4:], clean[4:]) and out[3].isnan().all()


def test_rows_are_independent_and_calls_repeat():
    """A row's bits: the same in every call, and whatever the other rows hold."""
    import torch
    for lens, rows in (([700, 90], [9, 9]), ([9000], [3]), ([300] * 40, [129] * 40)):
        batch = Batch(lens, rows, 12, 2, 128)
        first = batch.run()
        assert torch.equal(first, batch.run())
        q = batch.q.clone()
        q[1::2] = 3.0
        assert torch.equal(batch.run(q=q)[0:sum(rows):2], first[0:sum(rows):2])


def test_strided_rows_and_untouched_elements():
    import torch
    batch = Batch([100, 33], [3, 2], 6, 2, 64)
    want = batch.run()
    wide = torch.randn((batch.q.shape[0], 10, 64), device="cuda").bfloat16()
    wide[:, 2:8] = batch.q
    out = torch.full((batch.q.shape[0], 9, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    batch.run(q=wide[:, 2:8], out=out[:, 1:7])
    assert torch.equal(out[:5, 1:7], want[:5]) and (out[:, 0] == 5).all() and (out[:, 7:] == 5).all() and (out[5:] == 5).all()


def test_large_scores_and_far_maxima():
    """Scores of several hundred whose largest comes first, last or in the middle."""
    batch = Batch([400, 400], [1, 7], 8, 2, 128, q_scale=30.0)
    batch.check(batch.run())


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_values_of_any_range(hd):
    """Groups without a range, narrow ones far from zero, wide ones, ones beside the smallest and the largest numbers, in both roles."""
    import torch
    import paper_2602_24174_amd as T
    rng = np.random.default_rng(hd)
    n = 70
    x = rng.normal(size=(2, n, 2, hd)).astype(np.float32)
    kinds = [lambda v: v * 0, lambda v: v * 0 + 5, lambda v: v * 0 - 0.3, lambda v: 1e4 + v * 1e-3, lambda v: -300 + v * 1e-9, lambda v: v * 1e-30, lambda v: v * 1e-39,
             lambda v: 1e-20 + v * 1e-39, lambda v: v * 1e-41, lambda v: v * 40 + 1000]
    for t in range(n):
        x[1, t] = kinds[t % len(kinds)](x[1, t].astype(np.float64)).astype(np.float32)
    x[0, 3::7] = x[0, 3::7] * 0 + 0.25
    x[0, 5::7] = 1 + x[0, 5::7] * 1e-6
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    one = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for first, last in ((0, 10), (0, n), (8, 9), (6, 7), (1, 2), (4, 5), (9, 10)):
        some = x[:, first:last]
        cache = dirty_cache(6, 2, hd)
        T.tasc_kv4_append(cache, *(torch.tensor(some[i]).cuda() for i in (0, 1)), slots[:last - first])
        q = torch.tensor(rng.normal(size=(2, 6, hd)).astype(np.float32)).bfloat16().cuda()
        out = torch.zeros_like(q)
        T.tasc_kv4_attention(cache, q, torch.arange(6, dtype=torch.int32, device="cuda")[None], one([0, 2]), one([last - first]), 2, n, hd ** -0.5, out)
        want, bound = OK.attention(q.float().cpu().numpy().astype(np.float64), OK.quantise(some[0]), OK.quantise(some[1]), 2, hd ** -0.5)
        # (bf16's smallest number is 2^-133: half of it more, and the weights' products end there)
        assert (np.abs(out.float().cpu().numpy() - want) <= bound + 2.0 ** -133 * 33).all(), (first, last)


def test_values_of_the_largest_numbers():
    import torch
    import paper_2602_24174_amd as T
    rng = np.random.default_rng(8)
    x = rng.normal(size=(2, 20, 2, 64)).astype(np.float32)
    x[1, 4:9] = 1e36 * x[1, 4:9]
    x[1, 9:12] = -3e37 * (1 + 1e-3 * x[1, 9:12])
    cache, slots = dirty_cache(2, 2, 64), torch.arange(20, dtype=torch.int32, device="cuda")
    T.tasc_kv4_append(cache, *(torch.tensor(t).cuda() for t in x), slots)
    q = torch.tensor(rng.normal(size=(16, 4, 64)).astype(np.float32)).bfloat16().cuda()
    out = torch.zeros_like(q)
    one = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    T.tasc_kv4_attention(cache, q, one([[0, 1]]), one([0, 16]), one([20]), 16, 20, 0.125, out)
    want, bound = OK.attention(q.float().cpu().numpy().astype(np.float64), OK.quantise(x[0]), OK.quantise(x[1]), 16, 0.125)
    assert (np.abs(out.float().cpu().numpy() - want) <= bound).all()


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB whose last pages are used."""
    import torch
    import paper_2602_24174_amd as T
    heads, hd = 8, 128
    pages = (5 << 30) // T.tasc_kv4_page_bytes(heads, hd)
    cache = T.Kv4Cache(pages, heads, hd)
    rng = np.random.default_rng(5)
    k, v = tokens(rng, 48, heads, hd, "bfloat16"), tokens(rng, 48, heads, hd, "bfloat16")
    table = torch.tensor([[pages - 1, 3, pages - 2]], dtype=torch.int32, device="cuda")
    slots = (table[0].repeat_interleave(16) * 16 + torch.arange(48, device="cuda") % 16).to(torch.int32)
    T.tasc_kv4_append(cache, k, v, slots)
    assert (read(cache, slots)[0] == held(k)).all()
    q = torch.tensor(rng.normal(size=(1, 8, hd)).astype(np.float32)).bfloat16().cuda()
    out = torch.zeros_like(q)
    one = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    T.tasc_kv4_attention(cache, q, table, one([0, 1]), one([48]), 1, 48, hd ** -0.5, out)
    want, bound = OK.attention(q.float().cpu().numpy().astype(np.float64), *(OK.quantise(x.float().cpu().numpy()) for x in (k, v)), 1, hd ** -0.5)
    assert (np.abs(out.float().cpu().numpy() - want) <= bound).all()


def test_refusals_by_the_binding():
    import torch
    import paper_2602_24174_amd as T
    batch = Batch([40], [1], 4, 2, 64)
    k = torch.zeros((3, 2, 64), device="cuda")
    slots = torch.zeros(3, dtype=torch.int32, device="cuda")
    for bad in (dict(k=k[:2]), dict(v=k.bfloat16()), dict(k=k.half(), v=k.half()), dict(slots=slots.long()), dict(k=k.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(T.TascError):
            T.tasc_kv4_append(batch.cache, **dict(dict(k=k, v=k, slots=slots), **bad))
    q = batch.q
    for bad in (dict(q=q.float()), dict(q=q[..., :32].contiguous(), out=q[..., :32].contiguous()), dict(out=q[:1]), dict(row_off=batch.row_off[:1]), dict(kv_len=batch.kv_len.long())):
        a = dict(dict(q=q, table=batch.table, row_off=batch.row_off, kv_len=batch.kv_len, max_rows=1, max_kv=40, scale=1.0, out=torch.empty_like(q)), **bad)
        with pytest.raises(T.TascError):
            T.tasc_kv4_attention(batch.cache, **a)
    with pytest.raises(T.TascError):
        T.Kv4Cache(4, 2, 64, pool=torch.zeros(100, dtype=torch.uint8, device="cuda"))
    for shape in ((0, 2, 64), (4, 2, 48), (4, 0, 64)):
        with pytest.raises(T.TascError):
            T.Kv4Cache(*shape)

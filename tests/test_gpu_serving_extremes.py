"""The serving operators at the ends of their ranges: the most sequences, rows and tokens of a vocabulary, hints that are far off."""
import numpy as np
import pytest

from oracle import kv4 as OK
from oracle import page_tables as OP
from test_gpu_accept_sampled import check
from test_gpu_kv4 import Batch, dirty_cache, held, tokens

pytestmark = pytest.mark.gpu


def one(*v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def test_attention_of_the_most_sequences():
    """65535 (sequence, KV head) pairs of a row each over one to three tokens, whose pages they share."""
    import torch
    import paper_2602_24174_amd as T
    rng = np.random.default_rng(1)
    for B, kvh, heads, hd in ((65535, 1, 2, 64), (21845, 3, 3, 32)):
        print(f"{B} sequences, {heads}/{kvh} x {hd}", flush=True)
        pages = 8
        cache = dirty_cache(pages, kvh, hd)
        k, v = tokens(rng, 3 * pages, kvh, hd, "bfloat16"), tokens(rng, 3 * pages, kvh, hd, "bfloat16")
        slots = torch.arange(3 * pages, dtype=torch.int32, device="cuda")
        T.tasc_kv4_append(cache, k, v, slots // 3 * 16 + slots % 3)
        page, length = rng.integers(0, pages, B), rng.integers(1, 4, B)
        dev = lambda x: torch.tensor(x.astype(np.int32), device="cuda")
        q = torch.tensor(rng.normal(size=(B, heads, hd)).astype(np.float32)).bfloat16().cuda()
        out = torch.full_like(q, 7.0)
        T.tasc_kv4_attention(cache, q, dev(page)[:, None].contiguous(), torch.arange(B + 1, dtype=torch.int32, device="cuda"), dev(length), 1, 3, hd ** -0.5, out)
        got, x = out.float().cpu().numpy(), q.float().cpu().numpy().astype(np.float64)
        kq, vq = (OK.quantise(t.float().cpu().numpy()) for t in (k, v))
        first = held(v)[page * 3].repeat(heads // kvh, 1)
        alone = length == 1                                   # a row that sees one token gives its value
        assert (np.abs(got - first)[alone] <= 2.0 ** -7 * np.abs(first[alone]) + 2.0 ** -20).all()
        for b in rng.integers(0, B, 200).tolist() + [0, B - 1]:
            seen = slice(3 * page[b], 3 * page[b] + length[b])
            want, bound = OK.attention(x[b:b + 1], tuple(t[seen] for t in kq), tuple(t[seen] for t in vq), 1, hd ** -0.5)
            assert (np.abs(got[b] - want[0]) <= bound[0]).all(), b


def test_hints_that_are_far_off():
    """max_kv sizes the grid: the results hold whatever it says, and so does what a row behind it sees."""
    for lens, rows, heads, hd in (([2050, 40, 700], [9, 3, 1], 12, 128), ([5000], [1], 4, 64), ([300] * 50, [90] * 50, 12, 64)):
        batch = Batch(lens, rows, heads, 2, hd, seed=4)
        for hint in (1, 33, max(lens), 40000, 2 ** 31 - 1):
            print(f"tokens {lens[:3]}, max_kv {hint}", flush=True)
            if len(lens) < 50 or hint in (1, 2 ** 31 - 1):
                out = batch.run(max_kv=hint)
                few = Batch.__new__(Batch)
                few.__dict__.update(batch.__dict__)
                few.n = batch.n[:3]
                got = out.float().cpu().numpy()
                q = batch.q.float().cpu().numpy().astype(np.float64)
                for b, n in enumerate(few.n):
                    at = slice(batch.off[b], batch.off[b + 1])
                    want, bound = OK.attention(q[at], batch.k[b], batch.v[b], n, batch.scale)
                    assert (np.abs(got[at] - want) <= bound).all(), (hint, b)


def test_page_tables_of_the_most_sequences():
    import torch
    import paper_2602_24174_amd as T
    rng = np.random.default_rng(2)
    B, cols = 1 << 20, 2
    lens = rng.integers(0, 33, B)
    rows = np.minimum(rng.integers(0, 3, B), lens)
    hold = rng.integers(0, 2, B)
    lens[::1000], rows[7::1000] = 40, 33                      # too long for the table; more rows than tokens
    want_table = np.full((B, cols), -1).tolist()
    ask = int(np.maximum(-(-lens // 16) - hold, 0).sum())
    free = rng.permutation(ask)[:ask - 5000]
    cap = int(rows.sum()) + 9
    dev = lambda x: torch.tensor(np.asarray(x).astype(np.int32), device="cuda")
    table, pages, row_off = dev(want_table), dev(np.zeros(B)), dev(np.zeros(B + 1))
    slots, summary = dev(np.zeros(cap)), one(0, 0, 0)
    T.tasc_page_tables(dev(lens), dev(rows), dev(hold), dev(free), table, pages, row_off, slots, summary)
    want = OP.page_tables(lens.tolist(), rows.tolist(), hold.tolist(), free.tolist(), want_table, cap)
    assert (table.cpu().numpy() == np.array(want_table)).all()
    for g, w in zip((pages, row_off, slots, summary), want):
        assert (g.cpu().numpy() == np.array(w)).all()


def test_acceptance_of_the_most_rows():
    import torch
    rng = np.random.default_rng(3)
    for B, k, V in ((65535, 0, 3), (4369, 14, 40)):
        print(f"{B} x {k + 1} x {V}", flush=True)
        logits = torch.tensor(rng.normal(size=(B, k + 1, V)).astype(np.float32) * 4)
        drafts = logits[:, :k].argmax(-1).numpy().astype(np.int32)
        check(logits, drafts, None, None, rng.random((B, k + 1, 2)).astype(np.float32))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_acceptance_of_the_largest_vocabulary(dtype):
    import torch
    rng = np.random.default_rng(4)
    V, k = 1 << 24, 1
    logits = torch.tensor(rng.normal(size=(2, k + 1, V)).astype(np.float32) * 3).to(getattr(torch, dtype))
    logits[1, 0, V - 1] = 40.0
    drafts = np.array([[V - 2], [V - 1]], dtype=np.int32)
    u = np.array([[[0.5, 0.9999], [0.1, 0.5]], [[0.5, 0.3], [0.2, 1 - 2.0 ** -24]]], dtype=np.float32)
    check(logits, drafts, None, np.array([1.0, 0.8], dtype=np.float32), u)
    check(logits, drafts, np.full((2, k, V), 2.0 ** -24, dtype=np.float32), None, u)

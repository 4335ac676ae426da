"""The operators of a request's life together, eager and replayed: a prompt that several sequences continue, steps that grow, write and read their tables, draws
under filters, requests that end, pages that are given out again, a pool that is closed up.  At every step each sequence attends as one that has its
history to itself."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

LAYERS, HEADS, KV_HEADS, HD, PAGES, MAX_PAGES, BATCH, VOCAB = 2, 4, 2, 64, 64, 8, 8, 5000


class Server:
    """8 places for sequences over one pool, of 4-bit pages in two layers; the history of each place beside it, in plain tensors"""

    def __init__(self, seed):
        import torch
        import paper_2602_24174_amd as T
        self.T, self.torch, self.rng = T, torch, torch.Generator(device="cuda")
        self.rng.manual_seed(seed)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.page = T.tasc_kv4_page_bytes(KV_HEADS, HD)
        self.pool = torch.randint(0, 256, (LAYERS, PAGES * self.page), dtype=torch.uint8, device="cuda")
        self.caches = [T.Kv4Cache(PAGES, KV_HEADS, HD, pool=self.pool[j]) for j in range(LAYERS)]
        self.table = torch.full((BATCH, MAX_PAGES), -1, **i32)
        self.lens, self.new, self.pages = (torch.zeros(BATCH, **i32) for _ in range(3))
        self.row_off, self.slots, self.summary = torch.zeros(BATCH + 1, **i32), torch.zeros(BATCH * 40, **i32), torch.zeros(3, **i32)
        self.free, self.n_free = torch.arange(PAGES, **i32), PAGES
        self.history = [[(None, None)] * LAYERS for _ in range(BATCH)]

    def values(self, rows):
        return self.torch.randn((rows, KV_HEADS, HD), generator=self.rng, device="cuda").to(self.torch.bfloat16)

    def step(self, rows):
        """rows[b] new tokens for every place; their attention in each layer, and what it has to be"""
        T, torch = self.T, self.torch
        n = sum(rows)
        self.new.copy_(torch.tensor(rows, dtype=torch.int32))
        self.lens += self.new
        T.tasc_page_tables(self.lens, self.new, self.pages, self.free, self.table, self.pages_out(), self.row_off, self.slots, self.summary, n_free=self.n_free)
        self.pages.copy_(self.grown)
        assert self.summary[2] == 0
        self.n_free -= int(self.summary[1])
        self.free = self.free[int(self.summary[1]):].contiguous()
        outs = []
        for j, cache in enumerate(self.caches):
            k, v, q = self.values(n), self.values(n), torch.randn((n, HEADS, HD), generator=self.rng, device="cuda").to(torch.bfloat16)
            T.tasc_kv4_append(cache, k, v, self.slots[:n])
            at = 0
            for b, r in enumerate(rows):
                old = self.history[b][j]
                new = (k[at:at + r], v[at:at + r])
                self.history[b][j] = new if old[0] is None else tuple(torch.cat([o, x]) for o, x in zip(old, new))
                at += r
            outs.append((q, self.attend(cache, q, max(rows)), rows))
        for j, (q, out, _) in enumerate(outs):
            self.compare(j, q, out, rows)
        return outs

    def pages_out(self):
        self.grown = self.torch.zeros_like(self.pages)
        return self.grown

    def attend(self, cache, q, most):
        out = self.torch.zeros_like(q)
        self.T.tasc_kv4_attention(cache, q, self.table, self.row_off, self.lens, most, MAX_PAGES * 16, 0.125, out)
        return out

    def compare(self, j, q, out, rows):
        """A cache of its own for every sequence, filled with its history in one go, gives the same bits."""
        T, torch = self.T, self.torch
        at = 0
        for b, r in enumerate(rows):
            if r == 0:
                continue
            k, v = self.history[b][j]
            n = k.shape[0]
            assert n == int(self.lens[b])
            alone = T.Kv4Cache(MAX_PAGES, KV_HEADS, HD)
            slots = torch.arange(n, dtype=torch.int32, device="cuda")
            T.tasc_kv4_append(alone, k.contiguous(), v.contiguous(), slots)
            want, i32 = torch.zeros((r, HEADS, HD), dtype=torch.bfloat16, device="cuda"), dict(dtype=torch.int32, device="cuda")
            held = self.read(j, b, n)
            mine = [torch.empty((n, KV_HEADS, HD), device="cuda") for _ in range(2)]
            T.tasc_kv4_read(alone, slots, *mine)
            assert all(torch.equal(x, y) for x, y in zip(held, mine)), f"layer {j}, place {b}: the cache does not hold its history"
            T.tasc_kv4_attention(alone, q[at:at + r].contiguous(), torch.arange(MAX_PAGES, **i32)[None], torch.tensor([0, r], **i32), torch.tensor([n], **i32), max(rows), MAX_PAGES * 16,
                                 0.125, want)
            # (keys may be cut into other chunks: each side is off by a rounding of the weights and one of the result, half a step of bf16 each)
            assert (out[at:at + r].float() - want.float()).abs().max() <= 2 * 2.0 ** -8 * (mine[1].abs().max() + want.float().abs().max())
            at += r

    def read(self, j, b, n):
        torch = self.torch
        pos = torch.arange(n, device="cuda")
        slots = self.table[b, pos // 16] * 16 + (pos % 16).to(torch.int32)
        out = [torch.empty((n, KV_HEADS, HD), device="cuda") for _ in range(2)]
        self.T.tasc_kv4_read(self.caches[j], slots.contiguous(), *out)
        return out

    def fork(self, pairs, graph=False):
        T, torch = self.T, self.torch
        src, dst = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in zip(*pairs))
        frm, to, summary = torch.zeros_like(src), torch.zeros_like(src), torch.zeros(3, dtype=torch.int32, device="cuda")
        n = len(pairs)
        T.tasc_pages_fork(src, dst, self.lens, self.table, self.pages, self.free[:n].contiguous(), frm, to, summary)
        T.tasc_pages_copy(self.pool, self.page, PAGES, LAYERS, frm, to)
        assert summary[0] == n and summary[2] == 0
        self.free = self.free[n:].contiguous()             # (pages that were not needed turn up with the next list)
        self.n_free -= n
        for a, b in pairs:
            self.history[b] = list(self.history[a])

    def end(self, places):
        for b in places:
            self.lens[b] = self.pages[b] = 0
            self.history[b] = [(None, None)] * LAYERS
        free, summary = self.torch.zeros(PAGES, dtype=self.torch.int32, device="cuda"), self.torch.zeros(3, dtype=self.torch.int32, device="cuda")
        self.T.tasc_pages_free(self.table, self.pages, PAGES, free, summary)
        listed = {p for b in range(BATCH) for p in self.table[b, :int(self.pages[b])].tolist()}
        self.n_free = int(summary[0])
        assert self.n_free == PAGES - len(listed) and set(free[:self.n_free].tolist()) == set(range(PAGES)) - listed
        self.free = free[:self.n_free].contiguous()

    def compact(self):
        T, torch = self.T, self.torch
        frm, to, summary = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (PAGES // 2, PAGES // 2, 3))
        T.tasc_pages_compact(self.table, self.pages, PAGES, self.table, frm, to, summary)
        T.tasc_pages_copy(self.pool, self.page, PAGES, LAYERS, frm, to)
        used, moves, last = summary.tolist()
        assert used == last and max(int(self.table[b, :int(self.pages[b])].max()) for b in range(BATCH) if self.pages[b] > 0) == used - 1
        self.pool.view(LAYERS, PAGES, -1)[:, used:] = 0xA5    # (what is behind the live pages may be given back)
        self.free, self.n_free = torch.arange(used, PAGES, dtype=torch.int32, device="cuda"), PAGES - used
        return moves


@pytest.mark.parametrize("seed", [1, 2])
def test_a_days_requests(seed):
    s = Server(seed)
    s.step([37, 0, 0, 32, 0, 0, 1, 0])                      # three prompts: one ends inside a page, one with it, one token
    s.fork([(0, 1), (0, 2), (3, 4), (6, 5)])
    s.step([1, 1, 1, 1, 1, 1, 1, 0])
    s.step([3, 1, 2, 9, 1, 16, 1, 0])
    s.fork([(5, 7)])
    s.end([0, 3])                                           # their prompts' pages stay with 1, 2 and 4
    s.step([0, 2, 2, 0, 2, 2, 2, 2])
    s.step([20, 1, 1, 33, 1, 1, 1, 1])                      # new requests in the places, on pages that were given back
    s.end([1, 6])
    assert s.compact() > 0
    s.step([1, 0, 1, 1, 1, 1, 0, 1])
    s.fork([(2, 1), (7, 6)])
    s.step([1] * BATCH)
    s.end([0, 2, 3, 4, 5])
    s.compact()
    s.step([0, 4, 0, 0, 0, 0, 4, 4])


def test_a_recorded_step():
    """Tables, draws and free pages of a step recorded into a graph, with forked sequences, replayed while lengths and logits change"""
    import torch
    import paper_2602_24174_amd as T
    from oracle import filtered_sampling as OF
    from oracle import page_tables as OP
    from oracle import pages as OG
    i32 = dict(dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(3)
    B, cols, n_pages = 8, 12, 80
    lens, new, held, free = torch.zeros(B, **i32), torch.ones(B, **i32), torch.zeros(B, **i32), torch.arange(n_pages, **i32)
    table, pages, row_off, slots = torch.full((B, cols), -1, **i32), torch.zeros(B, **i32), torch.zeros(B + 1, **i32), torch.zeros(2 * B, **i32)
    logits, u, token, kept = torch.zeros((B, VOCAB), device="cuda"), torch.zeros(B, device="cuda"), torch.zeros(B, **i32), torch.zeros(B, **i32)
    k, p = torch.tensor([5, 50, 0, 0, 7, 1, 20, 0], **i32), torch.tensor([0.9, 1, 0.8, 0.5, 0.95, 1, 0.7, 0.99], device="cuda")
    left, count = torch.zeros(n_pages, **i32), torch.zeros(3, **i32)
    src, dst, frm, to = torch.tensor([0, 2], **i32), torch.tensor([1, 3], **i32), torch.zeros(2, **i32), torch.zeros(2, **i32)
    spare = torch.tensor([n_pages - 2, n_pages - 1], **i32)
    pool = torch.arange(3 * n_pages, **i32).repeat_interleave(4).view(3, n_pages, 4).contiguous()
    ws = [torch.empty(T.tasc_pages_workspace_bytes(n_pages), dtype=torch.uint8, device="cuda"), torch.empty(T.tasc_sample_workspace_bytes(B, VOCAB), dtype=torch.uint8, device="cuda")]

    def step():
        T.tasc_page_tables(lens, new, held, free, table, pages, row_off, slots, n_free=n_pages - 2)
        T.tasc_pages_fork(src, dst, lens, table, pages, spare, frm, to)
        T.tasc_pages_copy(pool, 16, n_pages, 3, frm, to)
        T.tasc_sample(logits, u, token, None, k, p, None, None, kept, ws[1])
        T.tasc_pages_free(table, pages, n_pages, left, count, ws[0])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        n = rng.integers(1, 100, B)
        n[1] = n[3] = 1
        x = (rng.standard_normal((B, VOCAB)) * 2).astype(np.float32)
        lens.copy_(torch.tensor(n, **i32))
        table.fill_(-1)
        logits.copy_(torch.tensor(x, device="cuda"))
        u.copy_(torch.tensor(rng.random(B).astype(np.float32), device="cuda"))
        before = pool.clone()
        graph.replay()
        torch.cuda.synchronize()
        want = [[-1] * cols for _ in range(B)]
        want_pages, _, want_slots, _ = OP.page_tables(n.tolist(), [1] * B, [0] * B, list(range(n_pages - 2)), want, 2 * B)
        want_lens = n.tolist()
        a, b, _ = OG.fork([0, 2], [1, 3], spare.tolist(), want_lens, want, want_pages)
        assert (table.tolist(), pages.tolist(), lens.tolist(), slots.tolist(), frm.tolist(), to.tolist()) == (want, want_pages, want_lens, want_slots, a, b)
        moved = before.tolist()
        OG.copies(moved, a, b)
        assert pool.tolist() == moved
        assert (left.tolist(), count.tolist()) == OG.free(want, want_pages, n_pages)
        for i in range(B):
            got = OF.sample(x[i], float(u[i]), 1.0, int(k[i]), np.float32(p[i].item()))
            assert (int(token[i]), int(kept[i])) == (got[0], got[2])

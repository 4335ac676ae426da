"""The operators of a serving step as a server runs them, one after the other without a host round trip: block tables and slots from the
lengths, the cache, attention over it, the verification of the drafts, and the lengths of the next step from what was accepted."""
import numpy as np
import pytest

from oracle import kv4 as OK
from oracle import page_tables as OP
from oracle import sampled_acceptance as OA

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS, HD, V, K = 6, 2, 64, 700, 3


class Server:
    """B sequences, K drafts a step.  Everything on the device, in buffers that a captured step can use again; a stream and workspaces of its own."""

    def __init__(self, B, pages, cols, seed, stream):
        import torch
        import paper_2602_24174_amd as T
        self.B, self.T, self.stream = B, T, stream
        i32 = dict(dtype=torch.int32, device="cuda")
        rng = np.random.default_rng(seed)
        self.cache = T.Kv4Cache(pages, KV_HEADS, HD)
        self.cache.pool.fill_(0xFF)
        self.lens, self.held, self.pages = torch.zeros(B, **i32), torch.zeros(B, **i32), torch.zeros(B, **i32)
        self.free = torch.tensor(rng.permutation(pages), **i32)
        self.table, self.row_off = torch.full((B, cols), -1, **i32), torch.zeros(B + 1, **i32)
        self.rows = B * (K + 1) + 3                                         # a padded batch
        self.slots, self.summary = torch.zeros(self.rows, **i32), torch.zeros(3, **i32)
        self.new, self.kv_len = torch.zeros(B, **i32), torch.zeros(B, **i32)
        self.at = torch.arange(pages, device="cuda")
        self.qkv = torch.zeros((self.rows, HEADS + 2 * KV_HEADS, HD), dtype=torch.bfloat16, device="cuda")
        self.out = torch.zeros((self.rows, HEADS, HD), dtype=torch.bfloat16, device="cuda")
        self.base, self.logits = torch.zeros((B, K + 1, V), device="cuda"), torch.zeros((B, K + 1, V), device="cuda")
        self.drafts, self.u = torch.zeros((B, K), **i32), torch.zeros((B, K + 1, 2), device="cuda")
        self.temperature = torch.tensor([0.0, 1.0, 0.7] * B, device="cuda")[:B].contiguous()
        self.accept_len, self.emitted = torch.zeros(B, **i32), torch.zeros((B, K + 1), **i32)
        self.logprob = torch.zeros((B, K + 1), device="cuda")
        self.max_kv = cols * 16
        self.ws = [torch.empty(max(n, 1), dtype=torch.uint8, device="cuda") for n in
                   (T.tasc_kv4_attention_workspace_bytes(B, self.rows, HEADS, KV_HEADS, HD, K + 1, self.max_kv), T.tasc_accept_sampled_workspace_bytes(B, K, V))]

    def fill(self, seed, new):
        """The step's inputs.  Sequences have `new` rows (0: none this step)."""
        import torch
        rng = np.random.default_rng(seed)
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        self.qkv.copy_(torch.tensor(rng.normal(size=self.qkv.shape).astype(np.float32)))
        x = rng.normal(size=self.base.shape).astype(np.float32) * 2
        x[..., 5] += 9
        self.base.copy_(torch.tensor(x))
        d = np.full((self.B, K), 5, dtype=np.int32)
        d[rng.random(d.shape) < 0.25] = 17
        self.drafts.copy_(torch.tensor(d))
        self.u.copy_(torch.tensor(rng.random(self.u.shape).astype(np.float32)))

    def step(self):
        import torch
        T, st = self.T, torch.cuda.current_stream().cuda_stream
        torch.add(self.lens, self.new, out=self.kv_len)
        T.tasc_page_tables(self.kv_len, self.new, self.held, self.free, self.table, self.pages, self.row_off, self.slots, self.summary, stream=st)
        self.held.copy_(self.pages)
        self.free.copy_(self.free[(self.at + self.summary[1]).clamp(max=self.at.numel() - 1)])      # (the tail repeats; the test has pages enough)
        k, v = self.qkv[:, HEADS:HEADS + KV_HEADS], self.qkv[:, HEADS + KV_HEADS:]
        T.tasc_kv4_append(self.cache, k, v, self.slots, stream=st)
        T.tasc_kv4_attention(self.cache, self.qkv[:, :HEADS], self.table, self.row_off, self.kv_len, K + 1, self.max_kv, HD ** -0.5, self.out, self.ws[0], stream=st)
        row = (self.row_off[:self.B, None] + torch.arange(K + 1, device="cuda")).clamp(max=self.rows - 1)
        torch.add(self.base, self.out[row.reshape(-1), 0, :1].float().reshape(self.B, K + 1, 1).expand(-1, -1, V) * self.base, out=self.logits)
        T.tasc_accept_sampled(self.logits, self.drafts, None, self.temperature, self.u, self.accept_len, self.emitted, self.logprob, self.ws[1], stream=st)
        self.lens.add_(torch.where(self.new > 0, self.accept_len + 1, 0))

    def state(self):
        return {n: getattr(self, n).clone() for n in ("lens", "held", "table", "row_off", "slots", "summary", "out", "logits", "accept_len", "emitted", "logprob", "free")}


class Check:
    """The same steps on the host."""

    def __init__(self, s):
        self.lens, self.held = [0] * s.B, [0] * s.B
        self.table, self.free = s.table.cpu().tolist(), s.free.cpu().tolist()
        self.k, self.v = ([np.zeros((0, KV_HEADS, HD), np.float32)] * s.B for _ in range(2))

    def step(self, s):
        new, x = s.new.tolist(), s.qkv.float().cpu().numpy()
        kv_len = [n + r for n, r in zip(self.lens, new)]
        pages, row_off, slots, summary = OP.page_tables(kv_len, new, self.held, self.free, self.table, s.rows)
        assert s.table.tolist() == self.table and s.pages.tolist() == pages and s.row_off.tolist() == row_off
        assert s.slots.tolist() == slots and s.summary.tolist() == summary and summary[2] == 0
        self.held, self.free = pages, self.free[summary[1]:]
        out, logits, drafts, u = (t.float().cpu().numpy() for t in (s.out, s.logits, s.drafts, s.u))
        for b, n in enumerate(new):
            if n == 0:
                continue
            rows = slice(row_off[b], row_off[b + 1])
            for held, at in ((self.k, HEADS), (self.v, HEADS + KV_HEADS)):
                held[b] = np.concatenate([held[b][:self.lens[b]], x[rows, at:at + KV_HEADS]])
            want, bound = OK.attention(x[rows, :HEADS].astype(np.float64), OK.quantise(self.k[b]), OK.quantise(self.v[b]), n, HD ** -0.5)
            assert (np.abs(out[rows] - want) <= bound).all()
            m, tokens, _ = OA.accept(logits[b], drafts[b].astype(int), None, float(s.temperature[b]), u[b])
            assert s.accept_len[b].item() == m and s.emitted[b].tolist() == tokens + [-1] * (K + 1 - len(tokens))
            self.lens[b] += m + 1
        assert s.lens.tolist() == self.lens


def rows_of(step, B):
    return [0 if (step + b) % 5 == 4 else K + 1 for b in range(B)]


@pytest.mark.parametrize("B, cols", [(1, 200), (7, 9)])
def test_steps_eager_and_replayed(B, cols):
    """A captured step, replayed with new inputs, does what the eager one does, which is what the host works out; two servers' steps, each with its
    stream, run at once, and eager work and synchronisations lie between the replays."""
    import torch
    torch.cuda.synchronize()
    eager = Server(B, 8 * B + 5, cols, 1, torch.cuda.current_stream())
    check = Check(eager)
    replayed = [Server(B, 8 * B + 5, cols, 1, torch.cuda.Stream()) for _ in range(2)]
    start = [{n: getattr(s, n).clone() for n in ("lens", "held", "free", "table")} for s in replayed]
    graphs = []
    for s in replayed:
        s.fill(99, rows_of(0, B))
        torch.cuda.synchronize()
        with torch.cuda.stream(s.stream):
            s.step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s.stream):
            s.step()
        graphs.append(g)
    for s, first in zip(replayed, start):
        for n, t in first.items():
            getattr(s, n).copy_(t)
    for step in range(6):
        print(f"step {step} of {B} sequences", flush=True)
        for s in (eager, *replayed):
            s.fill(step, rows_of(step, B))
        torch.cuda.synchronize()
        for s, g in zip(replayed, graphs):
            with torch.cuda.stream(s.stream):
                g.replay()
        eager.step()
        torch.cuda.synchronize()
        want = eager.state()
        for s in replayed:
            got = s.state()
            for n in want:
                if n in ("out", "logits", "accept_len", "emitted", "logprob"):
                    continue
                assert torch.equal(got[n], want[n]), n
            used = int(want["row_off"][-1])
            assert torch.equal(got["out"][:used], want["out"][:used])
            live = eager.new > 0
            for n in ("logits", "accept_len", "emitted", "logprob"):
                assert torch.equal(got[n][live], want[n][live]), n
        check.step(eager)

"""Sessions over a 4-bit cache.  Keys and values go through rounding to 16 numbers, where a last bit decides, so the oracle's forward takes what
the session's cache holds in place of its own keys and values: then its logits hold as they do for the other sessions (5e-2 on bf16 models of this
size).  What the first layer's cache holds is compared with the oracle's keys and values themselves."""
import numpy as np
import pytest

import workload as W
from oracle import kv4 as OK
from oracle import model as OM
from oracle import page_tables as OP

pytestmark = pytest.mark.gpu

BF16 = dict(dtype="bf16", n_layers=2, d_model=128, d_ffn=192, vocab=700, n_docs=800)
SHAPES = {
    "hd32": (dict(n_heads=6, n_kv_heads=2, head_dim=32, d_model=192), [37, 1, 5, 30], 32),
    "hd64": (dict(n_heads=4, n_kv_heads=2, head_dim=64), [300, 1, 2, 77, 150, 16], 40),
    "hd128": (dict(n_heads=4, n_kv_heads=1, head_dim=128), [260, 64, 65, 1], 17),
    # few rows a chunk, one sequence: no persistent kernel for it
    "one": (dict(n_heads=4, n_kv_heads=2, head_dim=64), [50], 4),
    # a prompt for every compute unit
    "many": (dict(n_heads=2, n_kv_heads=1, head_dim=64), [640 - (b * 53) % 600 for b in range(64)], 20),
    # long prompts: the first product's columns in one slice, waves with rows of their own
    "wide": (dict(n_heads=16, n_kv_heads=2, head_dim=128, d_model=2048, d_ffn=2048), [700 - b for b in range(16)], 64),
}


class Session4:
    def __init__(self, name, max_new=12, spare=0):
        import paper_2602_24174_amd as T
        shape, self.lens, self.max_rows = SHAPES[name]
        self.T, self.B = T, len(self.lens)
        self.cfg = W.get_config("cfg1").scaled(**dict(dict(BF16, batch=self.B), **shape))
        self.weights = W.make_model(self.cfg, W.make_corpus(self.cfg))
        rng = np.random.default_rng(3)
        self.prompts = [rng.integers(0, self.cfg.vocab, n).astype(np.int32) for n in self.lens]
        self.max_len = max(self.lens) + max_new + 2 * self.max_rows
        self.model = T.tasc_model_create(self.cfg, self.weights, self.max_len)
        self.max_new = max_new
        self.n_pages = sum(-(-(n + max_new + 2 * self.max_rows) // 16) for n in self.lens) + spare
        self.s = T.tasc_session_create_kv4(self.model, self.B, self.max_len, self.max_rows, self.n_pages)
        self.s._kv_pool.fill_(0xFF)                          # nothing relies on a cleared pool

    def prefill(self, prompts=None):
        prompts = prompts or self.prompts
        self.off = np.cumsum([0] + [len(p) for p in prompts]).astype(np.int64)
        self.T.tasc_session_prefill(self.model, self.s, np.concatenate(prompts), self.off, self.max_new)
        table = [[-1] * -(-self.max_len // 16) for _ in prompts]
        OP.page_tables([len(p) + self.max_new + 2 * self.max_rows for p in prompts], [0] * self.B, [0] * self.B, list(range(self.n_pages)), table, 0)
        self.table = table

    def held(self, b, n):
        """Keys and values of the first n tokens of a sequence, as the cache holds them: [layers, n, kv_heads, head_dim] each."""
        import torch
        c, T = self.cfg, self.T
        pos = np.arange(n)
        slots = torch.tensor(np.array(self.table[b])[pos // 16] * 16 + pos % 16, dtype=torch.int32, device="cuda")
        layer = self.n_pages * T.tasc_kv4_page_bytes(c.n_kv_heads, c.head_dim)
        out = [[], []]
        for l in range(c.n_layers):
            cache = T.Kv4Cache(self.n_pages, c.n_kv_heads, c.head_dim, pool=self.s._kv_pool[l * layer:(l + 1) * layer])
            k, v = (torch.zeros((n, c.n_kv_heads, c.head_dim), device="cuda") for _ in range(2))
            T.tasc_kv4_read(cache, slots, k, v)
            out[0].append(k.cpu().numpy())
            out[1].append(v.cpu().numpy())
        return np.stack(out[0]).astype(np.float64), np.stack(out[1]).astype(np.float64)


class HeldCache(OM.KVCache):
    """A cache that keeps what it was given."""

    class Kept(np.ndarray):
        def __setitem__(self, at, value):
            pass

    def __init__(self, k, v):
        self.k, self.v, self.length = k.view(self.Kept), v.view(self.Kept), 0


@pytest.mark.parametrize("name", list(SHAPES))
def test_logits_against_the_oracle(name):
    import torch
    x = Session4(name)
    T, k = x.T, 3
    assert T.tasc_session_kv4_bytes(x.model, x.n_pages) == x.cfg.n_layers * x.n_pages * T.tasc_kv4_page_bytes(x.cfg.n_kv_heads, x.cfg.head_dim)
    rng = np.random.default_rng(5)
    drafts = rng.integers(0, x.cfg.vocab, (x.B, k)).astype(np.int32)
    z = torch.zeros((x.B, k + 1, x.cfg.vocab), dtype=torch.float32, device="cuda")
    for again in range(2):                                   # the second prefill finds the first one's pages in use
        print(f"{name} prefill {again}", flush=True)
        x.prefill()
        T.tasc_verify_step(x.model, x.s, torch.from_numpy(drafts).cuda(), k, None, None, z)
        torch.cuda.synchronize()
        if again == 0:
            first = z.cpu().numpy()
    assert (z.cpu().numpy() == first).all()
    om = OM.OracleModel(x.cfg, x.weights)
    c = x.cfg
    for b in sorted({0, 1 % x.B, x.B // 2, x.B - 1}):
        n = x.lens[b]
        tokens = x.prompts[b].tolist() + [int(T.tasc_session_get_tokens(x.s, b)[n])] + drafts[b].tolist()
        kk, vv = x.held(b, n + 1 + k)
        want = om.forward(tokens, HeldCache(kk, vv))
        assert want[n - 1][tokens[n]] >= want[n - 1].max() - 0.1, "the committed token is not the target's argmax"
        worst = float(np.abs(first[b] - want[n:]).max())
        print(f"{name} sequence {b} ({n} tokens): max |logit - oracle| = {worst:.3e}", flush=True)
        assert worst <= 5e-2
        # the first layer's keys and values: h is rounded to bf16 (2^-8), then half a step and what rounding the scale takes (15 2^-8 steps)
        h = OM.rmsnorm(OM._to_f64(x.weights["embed"][tokens]), 1.0, c.rms_eps)
        for got, name_w in ((kk[0], "wk"), (vv[0], "wv")):
            w = om._layer(0, name_w)
            y, slack = ((a @ bb.T).reshape(-1, c.n_kv_heads, c.head_dim) for a, bb in ((h, w), (np.abs(h), np.abs(w))))
            slack = 2.0 ** -8 * 1.02 * slack
            if name_w == "wk":
                y = OM.rope(y, np.arange(len(tokens)), c.rope_theta)
                half = c.head_dim // 2
                slack = slack + np.concatenate([slack[..., half:], slack[..., :half]], -1)
            g = y.reshape(y.shape[:2] + (-1, min(c.head_dim, 64)))
            step = ((g.max(-1) - g.min(-1)) / 15)[..., None] + 2 * slack.reshape(g.shape).max(-1, keepdims=True) / 15
            slack = slack.reshape(g.shape)
            bound = 2 * slack.max(-1, keepdims=True) + step * (0.5 + 15 * 2.0 ** -8) + 2.0 ** -8 * np.abs(g.min(-1, keepdims=True))
            assert (np.abs(got.reshape(g.shape) - g) <= bound).all()


@pytest.mark.parametrize("name", ["hd32", "hd64", "hd128", "one", "many"])
def test_speculative_is_greedy(name):
    """Bit for bit: the same tokens with and without drafts, recorded steps and plain launches, one chain and several, and sampled at
    temperature 0; and in the same number of steps whatever ran before."""
    import torch
    x = Session4(name)
    T, c = x.T, x.cfg
    corpus = W.make_corpus(c)
    ng = T.tasc_ngram_build(corpus[0], corpus[1], c.vocab, c.n_max, c.p_min)
    x.prefill()
    out = torch.zeros((x.B, x.max_new), dtype=torch.int32, device="cuda")
    u = torch.rand((x.B, x.max_new, 2), device="cuda")

    def tokens(k, sampled=False):
        p = T.spec_params(k, c.lambda_q16, 1, 1)
        a = (x.model, ng if k else None, x.s, np.concatenate(x.prompts), x.off, x.max_new, p)
        T.tasc_generate_sampled(*a, u, out, torch.zeros(x.B, device="cuda")) if sampled else T.tasc_generate(*a, out)
        return out.cpu().numpy().copy()

    want = tokens(0)
    k = min(4, x.max_rows - 1)
    try:
        for graph, chains, kk in ((1, 0, k), (1, 0, 2), (0, 0, k), (1, 2, k), (0, 3, 0)):
            print(f"graph {graph}, chains {chains}, k {kk}", flush=True)
            T.tasc_config_set(T.TASC_CFG_STEP_GRAPH, graph)
            T.tasc_config_set(T.TASC_CFG_CHAINS, chains)
            assert (tokens(kk) == want).all()
    finally:
        T.tasc_config_set(T.TASC_CFG_STEP_GRAPH, 1)
        T.tasc_config_set(T.TASC_CFG_CHAINS, 0)
    assert (tokens(k, sampled=True) == want).all()


def test_a_prompt_is_its_own():
    """A prompt's cache and first token, bit for bit, whatever the prompts beside it."""
    x = Session4("hd64", spare=60)
    rng = np.random.default_rng(8)
    seen = []
    for others in ([1, 2, 77, 150, 16], [290, 30, 5, 9, 201]):
        x.prefill([x.prompts[0]] + [rng.integers(0, x.cfg.vocab, n).astype(np.int32) for n in others])
        seen.append((x.held(0, 300), x.T.tasc_session_get_tokens(x.s, 0).tolist()))
    assert seen[0][1] == seen[1][1] and all((a == b).all() for a, b in zip(seen[0][0], seen[1][0]))


def test_pages_by_lengths_and_refusals():
    import torch
    x = Session4("hd64")
    T = x.T
    x.prefill()                                              # exactly as many pages as these prompts need
    longer = list(x.prompts)
    longer[1] = np.zeros(40, dtype=np.int32)
    with pytest.raises(T.TascError) as e:
        x.prefill(longer)
    assert e.value.status == -2
    x.prefill()
    for bad in (0, -1, 1 << 27):
        with pytest.raises(T.TascError):
            T.tasc_session_create_kv4(x.model, x.B, x.max_len, x.max_rows, bad)
    small = T.tasc_session_kv4_bytes(x.model, 4)
    ws = torch.empty(T.tasc_session_workspace_bytes(x.model, 1, 64, 4), dtype=torch.uint8, device="cuda")
    pool, out = torch.empty(small, dtype=torch.uint8, device="cuda"), T.binding.C.c_void_p()
    make = lambda n, size: T.lib().tasc_session_create_kv4(x.model.handle, 1, 64, 4, n, pool.data_ptr(), size, ws.data_ptr(), ws.numel(), T.binding.C.byref(out))
    assert make(4, small - 1) == -2 and make(5, small) == -2
    cfg = W.get_config("cfg1")
    f32 = T.tasc_model_create(cfg, W.make_model(cfg), 128)
    assert T.tasc_session_kv4_bytes(f32, 10) == 0
    with pytest.raises(T.TascError):
        T.tasc_session_create_kv4(f32, 1, 128, 4, 10)


def test_model_bigram():
    """The vocabulary through a session over a 4-bit cache: a prompt of one token sees its own value only, so the successors are
    those of the oracle's logits with that token's key and value as held."""
    import torch
    x = Session4("one")
    T = x.T
    nxt = torch.full((x.cfg.vocab,), -1, dtype=torch.int32, device="cuda")
    T.tasc_model_bigram(x.model, x.s, nxt)
    got = nxt.cpu().numpy()
    om = OM.OracleModel(x.cfg, x.weights)
    for t in range(0, x.cfg.vocab, 37):
        z = om.forward([t], om.new_cache(1))[0]
        assert z[got[t]] >= z.max() - 0.5                    # (the oracle's value is not rounded to 16 numbers)

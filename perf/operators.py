"""The operators of a serving step over a 4-bit cache, as cases that can be timed and checked one by one.

A step of a server that decodes with drafts: the requests' lengths give block tables and slots on the GPU, the rows' keys and
values go to the cache in 4 bits, the rows attend to it, and the drafts are verified against the target's probabilities.

Kinds
  tables   `tasc_page_tables`: block tables grown from a list of free pages, the slots of the step's rows.
  cache    `tasc_kv4_append` of the rows' keys and values, and `tasc_kv4_read` of what the cache then holds for them.
  attend   `tasc_kv4_attention` of a step's or a prompt's rows over the cache.
  accept   `tasc_accept_sampled`: drafts against the target's probabilities, from given random numbers.

A case is a dict of plain values.  `prepare` makes what a program has in hand before the call, `run` is one pass, in the plain
form or through the library's entry points (`own`), `exact` the same in 64 bits, written apart from the plain form.

The cache's format: a token's head in groups of min(head_dim, 64) channels.  With lo and hi the least and the largest of a group's
values, scale = bf16((hi - lo) / 15) and low = bf16(lo), the steps in 32 bits; a value is held as the whole number in [0, 15]
nearest to (value - low) / scale (the even one of two; 0 where scale is 0) and stands for low + scale * number.
"""
import math
import types

import torch

own = False

PAGE = 16                # tokens of a page


def listed():
    return [
        # the decode loop's own bookkeeping: 64 sequences of up to 2,300 tokens, 9 rows each; launches are most of it
        {"name": "tables_step_b64", "kind": "tables", "batch": 64, "kv": 2300, "rows": 9, "fresh": 0.1, "short": False},
        # a large server: 4096 requests, a third of them new with whole prompts, tables of 2048 pages, too few free pages
        {"name": "tables_b4096", "kind": "tables", "batch": 4096, "kv": 16000, "rows": 600, "fresh": 0.33, "short": True},
        # a verify step's rows, out of the fused projection's bf16 rows
        {"name": "cache_step_b64", "kind": "cache", "rows": 576, "kv_heads": 2, "hd": 128, "dtype": "bf16", "fused": True},
        # a long prompt's keys and values as fp32
        {"name": "cache_prompt_f32", "kind": "cache", "rows": 16384, "kv_heads": 8, "hd": 128, "dtype": "f32", "fused": False},
        # interactive decoding: one sequence, one token, heads of 64; latency is most of it
        {"name": "attend_b1", "kind": "attend", "batch": 1, "kv": 700, "rows": 1, "heads": 9, "kv_heads": 3, "hd": 64},
        # the 1.5B shape's verify step: 9 rows over ragged contexts of up to 2,300 tokens
        {"name": "attend_15b_b64", "kind": "attend", "batch": 64, "kv": 2300, "rows": 9, "heads": 12, "kv_heads": 2, "hd": 128},
        # the 3B shape's verify step: many sequences, short contexts
        {"name": "attend_3b_b256", "kind": "attend", "batch": 256, "kv": 700, "rows": 5, "heads": 16, "kv_heads": 2, "hd": 128},
        # single tokens over long contexts, few sequences: the keys have to be split to fill the chip
        {"name": "attend_long_b2", "kind": "attend", "batch": 2, "kv": 131072, "rows": 1, "heads": 32, "kv_heads": 8, "hd": 128},
        # prompts: whole chunks of rows, causal
        {"name": "attend_prompt_b4", "kind": "attend", "batch": 4, "kv": 2500, "rows": 2048, "heads": 12, "kv_heads": 2, "hd": 128},
        # interactive decoding: 9 rows of the 135M shape's vocabulary
        {"name": "accept_b1", "kind": "accept", "batch": 1, "k": 8, "vocab": 49152, "dtype": "f32", "probs": False},
        # a drafting model's whole distributions beside the target's bf16 logits
        {"name": "accept_probs_b32", "kind": "accept", "batch": 32, "k": 6, "vocab": 151936, "dtype": "bf16", "probs": True},
        # the 3B shape's verify step, drafts without probabilities: 1280 rows of fp32 logits, the largest case
        {"name": "accept_b256", "kind": "accept", "batch": 256, "k": 4, "vocab": 151936, "dtype": "f32", "probs": False},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tables", "cache", "attend", "attend", "attend", "accept", "accept"])
    if kind == "tables":
        return {"kind": kind, "batch": _log(rng, 1, 4096), "kv": _log(rng, 16, 16000), "rows": _log(rng, 1, 600), "fresh": round(rng.random(), 2),
                "short": rng.random() < 0.3}
    if kind == "cache":
        hd = rng.choice([32, 64, 128])
        return {"kind": kind, "rows": _log(rng, 1, 16384), "kv_heads": rng.randint(1, 8), "hd": hd, "dtype": rng.choice(["bf16", "f32"]),
                "fused": rng.random() < 0.5}
    if kind == "accept":
        vocab = _log(rng, 500, 151936)
        k = rng.randint(0, 8)
        return {"kind": kind, "batch": _log(rng, 1, 128), "k": k, "vocab": vocab, "dtype": rng.choice(["bf16", "f32"]),
                "probs": k > 0 and rng.random() < 0.4}
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 6, 7, 8])
    hd = rng.choice([32, 64, 128])
    rows = rng.choice([1, rng.randint(2, 16), _log(rng, 17, 1500)])
    kv = _log(rng, max(rows, 1), 60000)
    batch = _log(rng, 1, 256)
    # no more score products than the prompts' case, no more keys than the long one, plain or not
    most = max(1, min(int(2e8 / (heads * rows * kv)), int(2.5e8 / (kv_heads * kv * hd))))
    if rows * kv * heads > 2e8:
        kv = max(rows, int(2e8 / (rows * heads)))
    return {"kind": kind, "batch": min(batch, most), "kv": kv, "rows": rows, "heads": heads, "kv_heads": kv_heads, "hd": hd}


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 64 + stream)
    return g


def _ints(g, lo, hi, n):                                   # in [lo, hi]
    return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int32)


def _lengths(case, g):
    """Tokens that the sequences hold after the step, and how many of them are the step's rows: ragged, the largest among them."""
    B, kv, rows = case["batch"], case["kv"], case["rows"]
    new = torch.full((B,), rows, dtype=torch.int32, device="cuda") if rows <= 16 else _ints(g, max(1, rows // 2), rows, B)
    lens = torch.maximum(_ints(g, max(1, kv // 2), kv, B), new)
    lens[0] = max(kv, rows)
    return lens, new


def _values(g, rows, heads, hd, dtype):
    """Keys or values of tokens: normal, with a few channels of larger range, as rotated keys have them."""
    x = torch.randn((rows, heads, hd), generator=g, device="cuda", dtype=torch.float32)
    x[..., 3::29] *= 4.0
    return x.to(dtype)


def _kv_of(case, seed, n_tokens):
    """(k, v) of all tokens of the sequences, bf16 [tokens, kv_heads, hd]."""
    return [_values(_gen(seed, 8 + i), n_tokens, case["kv_heads"], case["hd"], torch.bfloat16) for i in range(2)]


def _attend_inputs(case, seed):
    g = _gen(seed, 1)
    lens, new = _lengths(case, g)
    pages = (lens + PAGE - 1) // PAGE
    B, cols = case["batch"], int((max(case["kv"], case["rows"]) + PAGE - 1) // PAGE)
    n_pages = int(pages.sum())
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, cols), -1, dtype=torch.int32, device="cuda")
    first = torch.cumsum(pages, 0) - pages
    col = torch.arange(cols, device="cuda")[None, :]
    live = col < pages[:, None]
    table[live] = order[(first[:, None] + col)[live]]
    # every token of every sequence, sequence by sequence, and the slot it lies in
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), lens.long())
    start = torch.cumsum(lens, 0) - lens
    pos = torch.arange(seq.numel(), device="cuda") - start[seq]
    slots = (table[seq, pos // PAGE].long() * PAGE + pos % PAGE).to(torch.int32)
    row_off = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    row_off[1:] = torch.cumsum(new, 0)
    # as many rows as the step has room for: those behind the last sequence's are a padded batch's
    q = torch.randn((B * case["rows"], case["heads"], case["hd"]), generator=g, device="cuda").to(torch.bfloat16)
    return lens, new, table, slots, row_off, q, n_pages


def _accept_inputs(case, seed):
    g = _gen(seed, 2)
    B, k, V = case["batch"], case["k"], case["vocab"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    # a target that has learnt its task: a few likely tokens in each row over a wide floor
    logits = torch.randn((B, k + 1, V), generator=g, device="cuda", dtype=torch.float32) * 1.5
    likely = torch.randint(0, V, (B, k + 1, 8), generator=g, device="cuda")
    lift = torch.rand((B, k + 1, 8), generator=g, device="cuda") * 4.0 + 11.0
    logits.scatter_(2, likely, lift)
    logits = logits.to(dtype)
    probs = None
    if case["probs"]:
        noisy = logits[:, :k].float() + torch.randn((B, k, V), generator=g, device="cuda") * 0.5
        probs = torch.softmax(noisy, -1)
        drafts = torch.multinomial(probs.reshape(B * k, V), 1, generator=g).reshape(B, k).to(torch.int32) if k else torch.zeros((B, 0), dtype=torch.int32, device="cuda")
    else:
        drafts = torch.argmax(logits[:, :k], -1).to(torch.int32) if k else torch.zeros((B, 0), dtype=torch.int32, device="cuda")
        other = torch.rand((B, k), generator=g, device="cuda") < 0.15
        drafts = torch.where(other, likely[:, :k, 0].to(torch.int32), drafts)
    if k > 2 and not case["probs"]:
        drafts[::7, k - 1] = -1                            # some sequences have fewer drafts
    temperature = torch.full((B,), 0.8, device="cuda")
    temperature[1::5] = 0.0                                # some are decoded greedily
    temperature[2::5] = 1.0
    u = torch.rand((B, k + 1, 2), generator=g, device="cuda")
    return logits.contiguous(), drafts.contiguous(), probs, temperature, u


def _tables_inputs(case, seed):
    g = _gen(seed, 3)
    B = case["batch"]
    cols = 2 * ((case["kv"] + case["rows"] + PAGE - 1) // PAGE) + 1
    new = _ints(g, 1, case["rows"], B) if case["rows"] > 16 else torch.full((B,), case["rows"], dtype=torch.int32, device="cuda")
    fresh = torch.rand(B, generator=g, device="cuda") < case["fresh"]
    had = torch.where(fresh, torch.zeros_like(new), _ints(g, 1, case["kv"], B))
    lens = had + new
    held = (had + PAGE - 1) // PAGE
    n_held = int(held.sum())
    ask = int(((lens + PAGE - 1) // PAGE - held).clamp(min=0).sum())
    n_free = max(1, ask * 3 // 4 if case["short"] else ask + 100)
    order = torch.randperm(n_held + n_free, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, cols), -1, dtype=torch.int32, device="cuda")
    live = torch.arange(cols, device="cuda")[None, :] < held[:, None]
    table[live] = order[:n_held]
    return lens, new, held, order[n_held:].contiguous(), table, B * case["rows"] + 5


def _cache_inputs(case, seed):
    g = _gen(seed, 4)
    rows, h, hd = case["rows"], case["kv_heads"], case["hd"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    if case["fused"]:                                      # rows of a fused projection: queries, keys, values
        qkv = torch.cat([_values(g, rows, 2 * h, hd, dtype), _values(g, rows, h, hd, dtype), _values(g, rows, h, hd, dtype)], 1)
        k, v = qkv[:, 2 * h:3 * h], qkv[:, 3 * h:]
    else:
        k, v = _values(g, rows, h, hd, dtype), _values(g, rows, h, hd, dtype)
    n_pages = (rows + PAGE - 1) // PAGE + 3
    slots = torch.randperm(n_pages * PAGE, generator=g, device="cuda")[:rows].to(torch.int32)
    slots[rows // 2::97] = -1                              # rows of a padded batch
    return k, v, slots, n_pages


# ------------------------------------------------------------------------------------------------ what a program has in hand
def prepare(case, seed):
    s = types.SimpleNamespace(case=case)
    dev = dict(device="cuda")
    if own:
        import paper_2602_24174_amd as T
        s.T = T
    if case["kind"] == "tables":
        s.lens, s.new, s.held, s.free, s.table, cap = _tables_inputs(case, seed)
        B = case["batch"]
        s.pages = torch.zeros(B, dtype=torch.int32, **dev)
        s.row_off = torch.zeros(B + 1, dtype=torch.int32, **dev)
        s.slots = torch.zeros(cap, dtype=torch.int32, **dev)
        s.summary = torch.zeros(3, dtype=torch.int32, **dev)
    elif case["kind"] == "cache":
        s.k, s.v, s.slots, n_pages = _cache_inputs(case, seed)
        if own:
            s.cache = s.T.Kv4Cache(n_pages, case["kv_heads"], case["hd"])
            s.k_out = torch.empty((case["rows"], case["kv_heads"], case["hd"]), dtype=torch.float32, **dev)
            s.v_out = torch.empty_like(s.k_out)
    elif case["kind"] == "attend":
        s.lens, s.new, s.table, slots, s.row_off, s.q, n_pages = _attend_inputs(case, seed)
        k, v = _kv_of(case, seed, slots.numel())
        s.scale = 1.0 / math.sqrt(case["hd"])
        s.max_rows, s.max_kv = case["rows"], max(case["kv"], case["rows"])
        if own:                                            # the cache that the steps before have filled
            s.cache = s.T.Kv4Cache(n_pages, case["kv_heads"], case["hd"])
            s.T.tasc_kv4_append(s.cache, k, v, slots)
            s.out = torch.zeros_like(s.q)
            s.ws = torch.empty(s.T.tasc_kv4_attention_workspace_bytes(case["batch"], s.q.shape[0], case["heads"], case["kv_heads"], case["hd"], s.max_rows,
                                                                      s.max_kv), dtype=torch.uint8, **dev)
        else:                                              # the same pages, a byte a value
            shape = (n_pages * PAGE, case["kv_heads"], case["hd"])
            s.plain = []
            for x in (k, v):
                code, scale, low = _quantise(x)
                s.plain.append([torch.zeros((n_pages * PAGE,) + t.shape[1:], dtype=t.dtype, **dev).index_copy_(0, slots.long(), t) for t in (code, scale, low)])
                assert s.plain[-1][0].shape == shape
    else:
        s.logits, s.drafts, s.probs, s.temperature, s.u = _accept_inputs(case, seed)
        B, k = case["batch"], case["k"]
        if own:
            s.accept_len = torch.zeros(B, dtype=torch.int32, **dev)
            s.emitted = torch.zeros((B, k + 1), dtype=torch.int32, **dev)
            s.logprob = torch.zeros((B, k + 1), dtype=torch.float32, **dev)
            s.ws = torch.empty(s.T.tasc_accept_sampled_workspace_bytes(B, k, case["vocab"]), dtype=torch.uint8, **dev)
    return s


def run(s):
    kind = s.case["kind"]
    if kind == "tables":
        if not own:
            return _plain_tables(s)
        s.T.tasc_page_tables(s.lens, s.new, s.held, s.free, s.table, s.pages, s.row_off, s.slots, s.summary)
        return [s.table, s.pages, s.row_off, s.slots, s.summary]
    if kind == "cache":
        if not own:
            return [_plain_round_trip(x, s.slots) for x in (s.k, s.v)]
        s.T.tasc_kv4_append(s.cache, s.k, s.v, s.slots)
        s.T.tasc_kv4_read(s.cache, s.slots, s.k_out, s.v_out)
        return [s.k_out, s.v_out]
    if kind == "attend":
        if not own:
            return _plain_attention(s)
        s.T.tasc_kv4_attention(s.cache, s.q, s.table, s.row_off, s.lens, s.max_rows, s.max_kv, s.scale, s.out, s.ws)
        return s.out
    if not own:
        return _plain_accept(s)
    s.T.tasc_accept_sampled(s.logits, s.drafts, s.probs, s.temperature, s.u, s.accept_len, s.emitted, s.logprob, s.ws)
    return [s.accept_len, s.emitted, s.logprob]


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_tables(s):
    cols = s.table.shape[1]
    need = (s.lens + PAGE - 1) // PAGE
    fits = (s.new >= 0) & (s.new <= s.lens) & (need <= cols) & (s.held >= 0) & (s.held <= cols)
    ask = torch.where(fits, (need - s.held).clamp(min=0), torch.zeros_like(need))
    end = torch.cumsum(ask, 0)
    granted = fits & ((ask == 0) | (end <= s.free.numel()))
    col = torch.arange(cols, device="cuda")[None, :]
    new_page = granted[:, None] & (col >= s.held[:, None]) & (col < need[:, None])
    source = (end - ask)[:, None] + col - s.held[:, None]
    s.table.copy_(torch.where(new_page, s.free[source.clamp(0, s.free.numel() - 1)], s.table))
    s.pages.copy_(torch.where(granted, torch.maximum(need, s.held), s.held))
    rows = s.new.clamp(min=0)
    s.row_off[1:] = torch.cumsum(rows, 0)
    i = torch.arange(s.slots.numel(), device="cuda")
    seq = torch.searchsorted(s.row_off[1:].contiguous(), i.to(torch.int32), right=True)
    real = seq < s.lens.numel()
    seq = seq.clamp(max=s.lens.numel() - 1)
    pos = s.lens[seq] - s.new[seq] + (i - s.row_off[seq])
    page = s.table[seq, (pos // PAGE).clamp(0, cols - 1)]
    s.slots.copy_(torch.where(real & granted[seq], page * PAGE + pos % PAGE, torch.full_like(page, -1)))
    s.summary[0] = s.row_off[-1]
    s.summary[1] = torch.where(granted, end, torch.zeros_like(end)).max()
    s.summary[2] = (~granted).sum()
    return [s.table, s.pages, s.row_off, s.slots, s.summary]


def _quantise(x):
    """(whole numbers uint8 [rows, heads, hd], scale, low bf16 [rows, heads, groups]); the quotient in 64 bits: a value at a border
    must fall on its own side."""
    rows, heads, hd = x.shape
    group = min(hd, 64)
    g = x.float().reshape(rows, heads, hd // group, group)
    lo, hi = g.amin(-1), g.amax(-1)
    scale, low = ((hi - lo) / 15.0).to(torch.bfloat16), lo.to(torch.bfloat16)
    code = torch.empty((rows, heads, hd), dtype=torch.uint8, device=x.device)
    for at in range(0, rows, 1 << 15):                     # a slice at a time: 64 bits of long contexts are many bytes
        part = slice(at, at + (1 << 15))
        sc = scale[part].double()[..., None]
        n = torch.round((g[part].double() - low[part].double()[..., None]) / torch.where(sc == 0, torch.ones_like(sc), sc)).clamp(0, 15)
        code[part] = torch.where(sc == 0, torch.zeros_like(n), n).to(torch.uint8).reshape(-1, heads, hd)
    return code, scale, low


def _stands_for(code, scale, low):
    group = min(code.shape[-1], 64)
    c = code.float().unflatten(-1, (-1, group))
    return (c * scale.float()[..., None] + low.float()[..., None]).flatten(-2)


def _plain_round_trip(x, slots):
    return torch.where((slots >= 0)[:, None, None], _stands_for(*_quantise(x)), torch.zeros((), device="cuda"))


def _plain_attention(s):
    c = s.case
    B, H, G, hd = c["batch"], c["heads"], c["kv_heads"], c["hd"]
    R, L = s.max_rows, s.table.shape[1] * PAGE
    page = s.table.long().clamp(min=0)
    slot = (page[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")).reshape(B, L)
    out = torch.zeros_like(s.q)
    i, j = torch.arange(R, device="cuda"), torch.arange(L, device="cuda")
    live = i[None, :] < s.new[:, None]                                        # [B, R]
    row = (s.row_off[:-1, None] + i).clamp(max=s.q.shape[0] - 1)
    last = (s.lens - s.new)[:, None] + i                                      # the last key that a row sees
    step = max(1, int(2e9 / (H * R * L * 4 + G * L * hd * 16)))               # sequences at a time
    for b in range(0, B, step):
        e = min(B, b + step)
        k, v = (_stands_for(*(t[slot[b:e]] for t in x)) for x in s.plain)     # [n, L, G, hd]
        q = s.q[row[b:e]].float().reshape(e - b, R, G, H // G, hd).permute(0, 2, 1, 3, 4).reshape(e - b, G, R * (H // G), hd)
        score = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * s.scale                # [n, G, R * H / G, L]
        score = score.reshape(e - b, G, R, H // G, L)
        score.masked_fill_((j[None, None, :] > last[b:e, :, None])[:, None, :, None, :], -math.inf)
        top = score.amax(-1, keepdim=True)
        score.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
        total = score.sum(-1, keepdim=True)
        o = torch.matmul(score.reshape(e - b, G, R * (H // G), L), v.permute(0, 2, 1, 3).contiguous()).reshape(e - b, G, R, H // G, hd)
        o = torch.where(total > 0, o / torch.where(total > 0, total, torch.ones_like(total)), torch.zeros_like(o))
        o = o.permute(0, 2, 1, 3, 4).reshape(e - b, R, H, hd).to(torch.bfloat16)
        out[row[b:e][live[b:e]].long()] = o[live[b:e]]
    return out


def _plain_accept(s):
    B, k, V = s.case["batch"], s.case["k"], s.case["vocab"]
    b = torch.arange(B, device="cuda")
    x = s.logits.double()
    greedy = s.temperature == 0
    top = x.argmax(-1)                                                         # the lowest index of equal ones
    x = (x - x.amax(-1, keepdim=True)) / torch.where(greedy, torch.ones_like(s.temperature), s.temperature).double()[:, None, None]
    w = torch.exp(x)
    one = torch.zeros_like(w).scatter_(2, top[..., None], 1.0)
    w = torch.where(greedy[:, None, None], one, w)
    total = w.sum(-1)
    d = s.drafts.long()
    real = (d >= 0) & (d < V)
    safe = torch.where(real, d, torch.zeros_like(d))
    wd = w[:, :k].gather(2, safe[..., None])[..., 0]
    qd = torch.ones_like(wd) if s.probs is None else s.probs.gather(2, safe[..., None])[..., 0].double()
    ok = real & (s.u[:, :k, 0].double() * qd * total[:, :k] < wd)
    m = torch.cumprod(ok.int(), 1).sum(1) if k else torch.zeros(B, dtype=torch.int64, device="cuda")   # accepted drafts
    at = m.clamp(max=max(k - 1, 0))
    rejected = (m < k) & real[b, at] if k else torch.zeros(B, dtype=torch.bool, device="cuda")
    rest = w[b, m]
    if k:
        token = safe[b, at]
        if s.probs is None:
            left = rest.scatter(1, token[:, None], 0.0)
        else:
            left = (rest / total[b, m][:, None] - s.probs[b, at].double()).clamp(min=0)
        left = torch.where((left.sum(1) > 0)[:, None], left, rest)
        rest = torch.where(rejected[:, None], left, rest)
    cum = torch.cumsum(rest, 1)
    past = cum > s.u[b, m, 1].double()[:, None] * cum[:, -1:]
    pick = torch.where(past.any(1), past.int().argmax(1), V - 1 - (rest > 0).flip(1).int().argmax(1))
    i = torch.arange(k + 1, device="cuda")[None, :]
    drafted = torch.cat([safe, torch.zeros((B, 1), dtype=torch.int64, device="cuda")], 1)
    token = torch.where(i < m[:, None], drafted, pick[:, None])
    logp = torch.log(w.gather(2, token[..., None])[..., 0] / total)
    out = i <= m[:, None]
    return [m.to(torch.int32), torch.where(out, token, torch.full_like(token, -1)).to(torch.int32),
            torch.where(out, logp, torch.zeros_like(logp)).float()]


# ------------------------------------------------------------------------------------------------ in 64 bits, apart from the above
def exact(case, seed):
    return {"tables": _exact_tables, "cache": _exact_cache, "attend": _exact_attention, "accept": _exact_accept}[case["kind"]](case, seed)


def _exact_tables(case, seed):
    lens, new, held, free, table, cap = (t.tolist() if torch.is_tensor(t) else t for t in _tables_inputs(case, seed))
    cols, taken, refused, slots, row_off, pages = len(table[0]), 0, 0, [], [0], []
    asked = 0
    for b in range(case["batch"]):
        need = -(-lens[b] // PAGE)
        ask = max(0, need - held[b])
        good = need <= cols and (ask == 0 or asked + ask <= len(free))
        if need <= cols:
            asked += ask
        if good:
            for j in range(ask):
                table[b][held[b] + j] = free[asked - ask + j]
            taken = max(taken, asked)
        refused += not good
        pages.append(max(need, held[b]) if good else held[b])
        for pos in range(lens[b] - new[b], lens[b]):
            slots.append(table[b][pos // PAGE] * PAGE + pos % PAGE if good else -1)
        row_off.append(len(slots))
    n = len(slots)
    return [torch.tensor(t, dtype=torch.int32) for t in (table, pages, row_off, slots + [-1] * (cap - n), [n, taken, refused])]


def _exact_values(x):
    """What the cache holds of x [rows, heads, hd], in 64 bits."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for c in range(0, x.shape[-1], 64):
        part = x[..., c:c + 64].float()
        least, most = part.min(-1, keepdim=True).values, part.max(-1, keepdim=True).values
        step = ((most - least) / 15.0).bfloat16().double()
        base = least.bfloat16().double()
        n = ((part.double() - base) / step.where(step != 0, torch.full_like(step, math.inf))).round_().clamp_(0.0, 15.0)
        out[..., c:c + 64] = n.mul_(step).add_(base)
    return out


def _exact_cache(case, seed):
    k, v, slots, _ = _cache_inputs(case, seed)
    return [_exact_values(x) * (slots >= 0).double()[:, None, None] for x in (k, v)]


def _exact_attention(case, seed):
    lens, new, _, _, row_off, q, _ = _attend_inputs(case, seed)
    k, v = _kv_of(case, seed, int(lens.sum()))
    share = case["heads"] // case["kv_heads"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, r) in enumerate(zip(lens.tolist(), new.tolist())):
        first = int(row_off[b])
        seen = torch.arange(n, device="cuda")[None, :] <= torch.arange(n - r, n, device="cuda")[:, None]
        kb, vb = _exact_values(k[at:at + n]), _exact_values(v[at:at + n])
        for h in range(case["heads"]):
            z = (q[first:first + r, h].double() @ kb[:, h // share].t().contiguous()) / math.sqrt(case["hd"])
            out[first:first + r, h] = torch.softmax(z.masked_fill(~seen, -math.inf), -1) @ vb[:, h // share].contiguous()
        at += n
    return out


def _exact_accept(case, seed):
    logits, drafts, probs, temperature, u = _accept_inputs(case, seed)
    B, k, V = case["batch"], case["k"], case["vocab"]
    lens = torch.zeros(B, dtype=torch.int32)
    tokens = torch.full((B, k + 1), -1, dtype=torch.int32)
    logs = torch.zeros((B, k + 1), dtype=torch.float64)
    temps, wanted, chance = temperature.double().tolist(), drafts.tolist(), u.double().tolist()
    for b in range(B):
        for i in range(k + 1):
            z = logits[b, i].double()
            if temps[b] == 0:
                p = torch.zeros_like(z)
                p[int((z == z.max()).nonzero()[0])] = 1.0
                logp = p.log()
            else:
                logp = torch.log_softmax(z / temps[b], 0)
                p = logp.exp()
            d = wanted[b][i] if i < k else -1
            if 0 <= d < V:
                q = probs[b, i].double() if probs is not None else None
                if chance[b][i][0] * (1.0 if q is None else float(q[d])) < float(p[d]):
                    tokens[b, i], logs[b, i] = d, float(logp[d])
                    lens[b] += 1
                    continue
                if q is None:
                    r = p.clone()
                    r[d] = 0.0
                else:
                    r = (p - q).clamp_min(0.0)
                p = r if float(r.sum()) > 0 else p
            c = p.cumsum(0)
            t = int(torch.searchsorted(c, c[-1] * chance[b][i][1], right=True))
            if t >= V:
                t = int(p.nonzero()[-1])
            tokens[b, i], logs[b, i] = t, float(logp[t])
            break
    return [lens, tokens, logs]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] == "tables":
        rows = case["batch"] * case["rows"] * (0.5 if case["rows"] > 16 else 1)
        fresh_pages = case["batch"] * (rows / case["batch"] / PAGE + 0.5)
        return {"bytes": int(4 * (4 * case["batch"] + 2 * fresh_pages + 2 * rows)), "flops": int(4 * rows)}
    if case["kind"] == "cache":
        n = case["rows"] * case["kv_heads"]
        held = case["hd"] // 2 + 4 * max(1, case["hd"] // 64)
        return {"bytes": int(2 * n * (case["hd"] * ((2 if case["dtype"] == "bf16" else 4) + 4) + 2 * held)), "flops": int(2 * n * case["hd"] * 6)}
    if case["kind"] == "attend":
        tokens = case["batch"] * case["kv"] * 0.75
        rows = case["batch"] * case["rows"] * (0.75 if case["rows"] > 16 else 1)
        seen = case["kv"] * 0.75 - (0.375 * case["rows"] if case["rows"] > 16 else 0)
        held = 2 * case["kv_heads"] * (case["hd"] // 2 + 4 * max(1, case["hd"] // 64))
        return {"bytes": int(tokens * held + rows * case["heads"] * case["hd"] * 4), "flops": int(4 * rows * case["heads"] * case["hd"] * max(seen, 1))}
    n = case["batch"] * (case["k"] + 1) * case["vocab"]
    q = case["batch"] * case["vocab"] * 4 * (0.5 if case["probs"] else 0)
    return {"bytes": int(n * (2 if case["dtype"] == "bf16" else 4) + q), "flops": int(4 * n)}

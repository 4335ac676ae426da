"""The operators that a request's life needs beside a serving step's, as cases that can be timed and checked one by one.

A prompt is prefilled once and continued by several sequences that share its pages, their tokens are drawn under top-k, top-p and
min-p, requests end and leave their pages, and a pool that has become full of holes is closed up.

Kinds
  sample   `tasc_sample`: a token of each row of logits, from given random numbers.
  filter   `tasc_filter_logits`: the same filters as masked logits, for drafts that are verified against them.
  fork     `tasc_pages_fork` and `tasc_pages_copy`: sequences that continue others, in all layers of a pool.
  free     `tasc_pages_free`: the pages that no sequence lists.
  compact  `tasc_pages_compact` and `tasc_pages_copy`: the pages in use to the front of the pool.

A case is a dict of plain values.  `prepare` makes what a program has in hand before the call, `run` is one pass, in the plain
form or through the library's entry points (`own`), `exact` the same in 64 bits, written apart from the plain form.

The filters: a row's tokens by their logits, the largest first, the lowest index first among equal ones; w = exp((logit - largest) / temperature),
and 1 at the first alone where the temperature is 0.  With K = top_k (all tokens that are not masked where it is 0) and C the sums of w over the
places before each, a token is kept if its place is below K and, unless it is the first, C < top_p C_K (always, for top_p >= 1) and w >= min_p.
The token drawn is the lowest one up to which the kept weights sum to more than u times their total.
"""
import math
import types

import torch

own = False

PAGE = 16                # tokens of a page


def listed():
    return [
        # interactive decoding: one row of the 135M shape's vocabulary, the usual pair of filters; latency is most of it
        {"name": "sample_b1", "kind": "sample", "rows": 1, "vocab": 49152, "dtype": "f32", "filters": "k+p"},
        # one row of a large vocabulary, by mass alone: nothing bounds how many tokens are kept
        {"name": "sample_wide_b1", "kind": "sample", "rows": 1, "vocab": 151936, "dtype": "f32", "filters": "p"},
        # a batch of requests with settings of their own, bf16 logits
        {"name": "sample_b64", "kind": "sample", "rows": 64, "vocab": 151936, "dtype": "bf16", "filters": "mixed"},
        # all rows of a large server's step, the largest case
        {"name": "sample_b1280", "kind": "sample", "rows": 1280, "vocab": 151936, "dtype": "f32", "filters": "mixed"},
        # interactive decoding with drafts: 9 rows whose drafts are verified under the filters
        {"name": "filter_b1", "kind": "filter", "batch": 1, "k": 8, "vocab": 49152, "dtype": "f32", "filters": "k+p"},
        # the 1.5B shape's verify step: 64 sequences, 9 rows each
        {"name": "filter_b64", "kind": "filter", "batch": 64, "k": 8, "vocab": 151936, "dtype": "f32", "filters": "mixed"},
        # eight answers to one prompt, 4-bit pages of the 135M shape
        {"name": "fork_b8", "kind": "fork", "sources": 1, "copies": 7, "kv": 700, "layers": 30, "page": 3456},
        # a batch of prompts with 16 samples each, pages of 8 heads
        {"name": "fork_b512", "kind": "fork", "sources": 32, "copies": 15, "kv": 1000, "layers": 12, "page": 18432},
        # the decode loop's batch: what 64 sequences leave of a pool
        {"name": "free_b64", "kind": "free", "batch": 64, "kv": 2300, "spare": 0.3, "shared": 0.0},
        # a large server: 4096 requests that share their prompts' pages eight by eight
        {"name": "free_b4096", "kind": "free", "batch": 4096, "kv": 16000, "spare": 0.3, "shared": 0.5},
        # a small pool with a third of it in holes
        {"name": "compact_b16", "kind": "compact", "batch": 16, "kv": 700, "spare": 0.33, "shared": 0.0, "layers": 30, "page": 3456},
        # the 1.5B shape's layers: thousands of pages
        {"name": "compact_b64", "kind": "compact", "batch": 64, "kv": 900, "spare": 0.33, "shared": 0.25, "layers": 28, "page": 4608},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["sample", "sample", "sample", "filter", "filter", "fork", "free", "compact"])
    filters = rng.choice(["k", "p", "min", "k+p", "mixed", "none"])
    dtype = rng.choice(["bf16", "f32"])
    if kind == "sample":
        return {"kind": kind, "rows": _log(rng, 1, 700), "vocab": _log(rng, 500, 151936), "dtype": dtype, "filters": filters}
    if kind == "filter":
        return {"kind": kind, "batch": _log(rng, 1, 64), "k": rng.randint(0, 8), "vocab": _log(rng, 500, 151936), "dtype": dtype, "filters": filters}
    page = rng.choice([640, 1152, 2304, 3456, 4608, 9216, 18432])
    spare, shared = round(rng.uniform(0.02, 0.7), 2), rng.choice([0.0, round(rng.random(), 2)])
    if kind == "fork":
        sources, copies, kv = _log(rng, 1, 32), _log(rng, 1, 16), _log(rng, 1, 2000)
        layers = max(1, min(rng.randint(1, 36), int(4e8 / (sources * (kv / PAGE + copies + 1) * page))))
        return {"kind": kind, "sources": sources, "copies": copies, "kv": kv, "layers": layers, "page": page}
    if kind == "free":
        batch = _log(rng, 1, 4096)
        return {"kind": kind, "batch": batch, "kv": _log(rng, 16, 16000), "spare": spare, "shared": shared}
    batch, kv = _log(rng, 1, 128), _log(rng, 16, 2000)
    layers = max(1, min(rng.randint(1, 36), int(4e8 * (1 - spare) / (batch * (kv / PAGE + 1) * page))))
    return {"kind": kind, "batch": batch, "kv": kv, "spare": spare, "shared": shared, "layers": layers, "page": page}


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 64 + stream)
    return g


def _ints(g, lo, hi, n):                                   # in [lo, hi]
    return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int32)


def _between(g, lo, hi, n):
    return torch.rand(n, generator=g, device="cuda") * (hi - lo) + lo


def _logits(g, rows, vocab, dtype):
    """A few likely tokens in each row over a wide floor: most rows sure of what they say, a third of them not; some rows are masked to a part of
    the vocabulary."""
    x = torch.randn((rows, vocab), generator=g, device="cuda", dtype=torch.float32)
    x.mul_(1.5)
    likely = torch.randint(0, vocab, (rows, 8), generator=g, device="cuda")
    unsure = (torch.arange(rows, device="cuda") % 3 == 2)[:, None]
    lift = torch.rand((rows, 8), generator=g, device="cuda") * 4.0 + torch.where(unsure, 5.0, 11.0)
    x.scatter_(1, likely, lift)
    for r in range(3, rows, 8):
        x[r, torch.rand(vocab, generator=g, device="cuda") < 0.5] = -math.inf
        x[r, r % vocab] = 1.0
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _filters(g, kind, n):
    """(temperature, top_k, top_p, min_p), None for those that the program leaves out"""
    temperature = _between(g, 0.6, 1.1, n)
    top_k = _ints(g, 5, 200, n)
    top_p = _between(g, 0.8, 0.98, n)
    min_p = _between(g, 0.01, 0.2, n)
    if kind == "mixed":
        i = torch.arange(n, device="cuda") % 8
        temperature = torch.where(i == 5, torch.zeros_like(temperature), temperature)        # greedy ones among them
        top_k = torch.where((i == 0) | (i == 1) | (i == 4), top_k, torch.zeros_like(top_k))
        top_p = torch.where((i == 1) | (i == 2) | (i == 3) | (i == 4), top_p, torch.ones_like(top_p))
        min_p = torch.where((i == 4) | (i == 6), min_p, torch.zeros_like(min_p))
        return temperature, top_k, top_p, min_p
    return (temperature, top_k if "k" in kind else None, top_p if "p" in kind.split("+") else None, min_p if kind == "min" else None)


def _sample_inputs(case, seed):
    g = _gen(seed, 1)
    rows = case["rows"] if case["kind"] == "sample" else case["batch"] * (case["k"] + 1)
    per = 1 if case["kind"] == "sample" else case["k"] + 1
    logits = _logits(g, rows, case["vocab"], case["dtype"])
    filters = _filters(g, case["filters"], rows // per)
    u = torch.rand(rows, generator=g, device="cuda")
    return logits, filters, u, per


def _spread(g, lo, hi, n):
    """Lengths evenly spread over [lo, hi], in any order: pools of different inputs are of one size."""
    lens = torch.linspace(hi, lo, n, device="cuda", dtype=torch.float64).round().to(torch.int32)
    return lens[torch.randperm(n, generator=g, device="cuda")]


def _tables(g, lens, longest, n_pages, shared=0.0):
    """Tables of sequences of these lengths over pages anywhere in a pool; of each eight in a row, the later ones list a share of the first one's."""
    pages = (lens + PAGE - 1) // PAGE
    B, cols = lens.numel(), (longest + PAGE - 1) // PAGE + 2
    table = torch.full((B, cols), -1, dtype=torch.int32, device="cuda")
    col = torch.arange(cols, device="cuda")[None, :]
    live = col < pages[:, None]
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table[live] = order[:int(pages.sum())]
    if shared:
        first = torch.arange(B, device="cuda") // 8 * 8
        common = (torch.minimum(pages, pages[first]) * shared).to(torch.int32)
        table = torch.where(col < common[:, None], table[first], table)
    return table, pages.to(torch.int32)


def _pool(g, layers, n_pages, page):
    return torch.randint(-2 ** 63, 2 ** 63 - 1, (layers, n_pages, page // 8), generator=g, device="cuda").view(torch.uint8)


def _fork_inputs(case, seed):
    g = _gen(seed, 2)
    S, per, kv = case["sources"], case["copies"], case["kv"]
    B = S * (per + 1)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    at = torch.randperm(B, generator=g, device="cuda").to(torch.int32)
    src, dst = at[:S], at[S:]                              # the sequences that hold a prompt, and the free places beside them
    lens[src.long()] = _spread(g, max(1, kv // 2), kv, S)
    held = int(((lens + PAGE - 1) // PAGE).sum())
    table, pages = _tables(g, lens, kv, held + dst.numel())
    new = torch.ones(held + dst.numel(), dtype=torch.bool, device="cuda")
    new[table[table >= 0].long()] = False
    return lens, src.repeat_interleave(per), dst.contiguous(), table, pages, new.nonzero()[:, 0].to(torch.int32), held + dst.numel()


def _in_use(case, seed):
    """(table, pages, n_pages) of requests in the middle of a server's day"""
    g = _gen(seed, 3)
    lens = _spread(g, max(1, case["kv"] // 4), case["kv"], case["batch"])
    n_pages = max(1, int(int(((lens + PAGE - 1) // PAGE).sum()) / (1 - case["spare"])))
    return (*_tables(g, lens, case["kv"], n_pages, case["shared"]), n_pages)


# ------------------------------------------------------------------------------------------------ what a program has in hand
def prepare(case, seed):
    s = types.SimpleNamespace(case=case)
    i32 = dict(dtype=torch.int32, device="cuda")
    if own:
        import paper_2602_24174_amd as T
        s.T = T
    if case["kind"] in ("sample", "filter"):
        s.logits, s.filters, s.u, s.per = _sample_inputs(case, seed)
        rows = s.logits.shape[0]
        if own:
            s.ws = torch.empty(T.tasc_sample_workspace_bytes(rows, case["vocab"]), dtype=torch.uint8, device="cuda")
            s.kept = torch.zeros(rows, **i32)
            s.token, s.logprob = torch.zeros(rows, **i32), torch.zeros(rows, dtype=torch.float32, device="cuda")
            if case["kind"] == "filter":
                s.logits = s.logits.view(case["batch"], s.per, case["vocab"])
                s.kept = s.kept.view(case["batch"], s.per)
                s.out = torch.empty_like(s.logits)
    elif case["kind"] == "fork":
        s.lens, s.src, s.dst, s.table, s.pages, s.new, s.n_pages = _fork_inputs(case, seed)
        s.pool = _pool(_gen(seed, 4), case["layers"], s.n_pages, case["page"])
        s.copy_from, s.copy_to, s.summary = torch.zeros_like(s.dst), torch.zeros_like(s.dst), torch.zeros(3, **i32)
    else:
        s.table, s.pages, s.n_pages = _in_use(case, seed)
        s.summary = torch.zeros(3, **i32)
        if own:
            s.ws = torch.empty(T.tasc_pages_workspace_bytes(s.n_pages), dtype=torch.uint8, device="cuda")
        if case["kind"] == "free":
            s.free = torch.zeros(s.n_pages, **i32)
        else:
            s.pool = _pool(_gen(seed, 4), case["layers"], s.n_pages, case["page"])
            s.after = s.table.clone()
            s.copy_from, s.copy_to = torch.zeros(s.n_pages // 2 + 1, **i32), torch.zeros(s.n_pages // 2 + 1, **i32)
    return s


def run(s):
    kind = s.case["kind"]
    if kind == "sample":
        if not own:
            return _plain_sample(s, False)
        s.T.tasc_sample(s.logits, s.u, s.token, *s.filters, s.logprob, s.kept, s.ws)
        return [s.token, s.logprob, s.kept]
    if kind == "filter":
        if not own:
            return _plain_sample(s, True)
        s.T.tasc_filter_logits(s.logits, s.out, *s.filters, s.kept, s.ws)
        return [s.out, s.kept]
    if kind == "free":
        if not own:
            return _plain_free(s)
        s.T.tasc_pages_free(s.table, s.pages, s.n_pages, s.free, s.summary, s.ws)
        return [s.free, s.summary]
    if kind == "fork":
        if own:
            s.T.tasc_pages_fork(s.src, s.dst, s.lens, s.table, s.pages, s.new, s.copy_from, s.copy_to, s.summary)
            s.T.tasc_pages_copy(s.pool, s.case["page"], s.n_pages, s.case["layers"], s.copy_from, s.copy_to)
        else:
            _plain_fork(s)
        return [s.lens, s.table, s.pages, s.copy_from, s.copy_to, s.summary, s.pool]
    if own:
        s.T.tasc_pages_compact(s.table, s.pages, s.n_pages, s.after, s.copy_from, s.copy_to, s.summary, s.ws)
        s.T.tasc_pages_copy(s.pool, s.case["page"], s.n_pages, s.case["layers"], s.copy_from, s.copy_to)
    else:
        _plain_compact(s)
    return [s.after, s.copy_from, s.copy_to, s.summary, s.pool]


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_sample(s, masked):
    rows, V = s.logits.shape
    token, kept = (torch.empty(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    logprob = torch.empty(rows, dtype=torch.float32, device="cuda")
    out = torch.empty_like(s.logits) if masked else None
    per_row = [None if f is None else f.repeat_interleave(s.per)[:, None] for f in s.filters]
    step = max(1, int(2e7 / V))                            # rows at a time: 64 bits a logit, several times over
    for r in range(0, rows, step):
        part = slice(r, min(rows, r + step))
        temperature, top_k, top_p, min_p = (None if f is None else f[part] for f in per_row)
        x, order = torch.sort(s.logits[part].float(), dim=1, descending=True, stable=True)
        greedy = temperature == 0
        z = (x[:, :1].double() - x.double()) / torch.where(greedy, torch.ones_like(temperature), temperature).double()
        place = torch.arange(V, device="cuda")[None, :]
        w = torch.where(greedy, (place == 0).double(), torch.exp(-z))
        live = (x > -math.inf) & (~greedy | (place == 0))
        if top_k is not None:
            live &= (top_k <= 0) | (place < top_k)
        w = torch.where(live, w, torch.zeros_like(w))
        keep = live
        if top_p is not None:
            up = torch.cumsum(w, 1)
            before = torch.cat([torch.zeros_like(up[:, :1]), up[:, :-1]], 1)
            keep = keep & ((place == 0) | (top_p >= 1) | (before < top_p.double() * up[:, -1:]))
        if min_p is not None:
            keep = keep & ((place == 0) | (w >= min_p.double()))
        kept[part] = keep.sum(1, dtype=torch.int32)
        keep = torch.zeros_like(keep).scatter_(1, order, keep)
        if masked:
            out[part] = torch.where(keep, s.logits[part], torch.full_like(s.logits[part], -math.inf))
            continue
        w = torch.where(keep, torch.zeros_like(w).scatter_(1, order, w), torch.zeros_like(w))
        up = torch.cumsum(w, 1)
        past = (up > s.u[part].double()[:, None] * up[:, -1:]) & (w > 0)
        t = torch.where(past.any(1), past.int().argmax(1), V - 1 - (w > 0).flip(1).int().argmax(1))
        token[part] = t.to(torch.int32)
        logprob[part] = torch.log(w.gather(1, t[:, None])[:, 0] / w.sum(1)).float()
    return [out.view(s.case["batch"], s.per, V), kept.view(s.case["batch"], s.per)] if masked else [token, logprob, kept]


def _plain_fork(s):
    lens, cols = s.lens[s.src.long()], s.table.shape[1]
    need = (lens + PAGE - 1) // PAGE
    col = torch.arange(cols, device="cuda")[None, :]
    rows = s.table[s.src.long()]
    part = lens % PAGE != 0
    last = rows.gather(1, (need - 1).clamp(min=0).long()[:, None])[:, 0]
    s.copy_from.copy_(torch.where(part, last, torch.full_like(last, -1)))
    s.copy_to.copy_(torch.where(part, s.new, torch.full_like(s.new, -1)))
    rows = torch.where(part[:, None] & (col == need[:, None] - 1), s.new[:, None], rows)
    s.table[s.dst.long()] = torch.where(col < need[:, None], rows, s.table[s.dst.long()])
    s.lens[s.dst.long()] = lens
    s.pages[s.dst.long()] = need.to(torch.int32)
    s.summary[0] = s.dst.numel()
    s.summary[1] = part.sum()
    s.summary[2] = 0
    s.pool[:, s.copy_to[part].long()] = s.pool[:, s.copy_from[part].long()]


def _listed_pages(s):
    """(which pages any table lists, how many entries do)"""
    live = torch.arange(s.table.shape[1], device="cuda")[None, :] < s.pages[:, None]
    at = s.table[live].long()
    return torch.zeros(s.n_pages, dtype=torch.bool, device="cuda").index_fill_(0, at, True), live.sum()


def _plain_free(s):
    used, entries = _listed_pages(s)
    at = (~used).nonzero()[:, 0].to(torch.int32)
    s.free.fill_(-1)
    s.free[:at.numel()] = at
    s.summary[0] = at.numel()
    s.summary[1] = s.n_pages - at.numel()
    s.summary[2] = entries
    return [s.free, s.summary]


def _plain_compact(s):
    used, _ = _listed_pages(s)
    n = used.sum()
    page = torch.arange(s.n_pages, device="cuda")
    far = (used & (page >= n)).nonzero()[:, 0].flip(0)
    hole = (~used & (page < n)).nonzero()[:, 0]
    s.copy_from.fill_(-1)
    s.copy_to.fill_(-1)
    s.copy_from[:far.numel()] = far.to(torch.int32)
    s.copy_to[:far.numel()] = hole.to(torch.int32)
    now = page.clone()
    now[far] = hole
    live = torch.arange(s.table.shape[1], device="cuda")[None, :] < s.pages[:, None]
    s.after.copy_(torch.where(live, now[s.table.long().clamp(min=0)].to(torch.int32), s.after))
    s.summary[0] = n
    s.summary[1] = far.numel()
    s.summary[2] = n
    s.pool[:, hole] = s.pool[:, far]


# ------------------------------------------------------------------------------------------------ in 64 bits, apart from the above
def exact(case, seed):
    return {"sample": _exact_sample, "filter": _exact_sample, "fork": _exact_fork, "free": _exact_free, "compact": _exact_compact}[case["kind"]](case, seed)


def _exact_sample(case, seed):
    logits, filters, u, per = _sample_inputs(case, seed)
    temps, ks, ps, ms = (None if f is None else f.double().tolist() for f in filters)
    chance = u.double().tolist()
    tokens, logs, kept = [], [], []
    out = torch.full_like(logits, -math.inf, dtype=torch.float64) if case["kind"] == "filter" else None
    for r in range(logits.shape[0]):
        b = r // per
        row = logits[r].double()
        ids = torch.sort(row, descending=True, stable=True).indices
        if temps[b] == 0:
            ids = ids[:1]
        ids = ids[:int((row > -math.inf).sum())]
        if ks is not None and ks[b] > 0:
            ids = ids[:int(ks[b])]
        scaled = row[ids] / (temps[b] or 1.0)
        n = ids.numel()
        if ps is not None and ps[b] < 1:                   # the shortest run from the front with that share of the mass
            mass = torch.softmax(scaled, 0).cumsum(0)
            n = min(n, 1 + int((mass[:-1] < ps[b] * mass[-1]).sum()))
        if ms is not None and ms[b] > 0:
            n = min(n, max(1, int((scaled >= scaled[0] + math.log(ms[b])).sum())))
        ids = ids[:n].sort().values
        kept.append(n)
        if out is not None:
            out[r, ids] = row[ids]
            continue
        logp = torch.log_softmax(row[ids] / (temps[b] or 1.0), 0)
        mass = logp.exp().cumsum(0)
        at = min(int(torch.searchsorted(mass, mass[-1] * chance[r], right=True)), n - 1)
        tokens.append(int(ids[at]))
        logs.append(float(logp[at]))
    kept = torch.tensor(kept, dtype=torch.int32)
    if out is not None:
        return [out.view(case["batch"], per, -1), kept.view(case["batch"], per)]
    return [torch.tensor(tokens, dtype=torch.int32), torch.tensor(logs, dtype=torch.float64), kept]


def _exact_fork(case, seed):
    lens, src, dst, table, pages, new, n_pages = (t.tolist() if torch.is_tensor(t) else t for t in _fork_inputs(case, seed))
    pool = _pool(_gen(seed, 4), case["layers"], n_pages, case["page"])
    copy_from, copy_to = [], []
    for a, b, fresh in zip(src, dst, new):
        need = -(-lens[a] // PAGE)
        lens[b], pages[b] = lens[a], need
        table[b][:need] = table[a][:need]
        copy_from.append(-1)
        copy_to.append(-1)
        if lens[a] % PAGE:
            copy_from[-1], copy_to[-1] = table[a][need - 1], fresh
            table[b][need - 1] = fresh
            pool[:, fresh] = pool[:, copy_from[-1]]
    done = [len(src), sum(p >= 0 for p in copy_to), 0]
    return [torch.tensor(t, dtype=torch.int32) for t in (lens, table, pages, copy_from, copy_to, done)] + [pool]


def _exact_free(case, seed):
    table, pages, n_pages = _in_use(case, seed)
    free = set(range(n_pages))
    entries = 0
    for row, n in zip(table.tolist(), pages.tolist()):
        free.difference_update(row[:n])
        entries += n
    count = len(free)
    return [torch.tensor(sorted(free) + [-1] * (n_pages - count), dtype=torch.int32), torch.tensor([count, n_pages - count, entries], dtype=torch.int32)]


def _exact_compact(case, seed):
    table, pages, n_pages = _in_use(case, seed)
    pool = _pool(_gen(seed, 4), case["layers"], n_pages, case["page"])
    table, pages = table.tolist(), pages.tolist()
    used = {p for row, n in zip(table, pages) for p in row[:n]}
    moves = list(zip(sorted((p for p in used if p >= len(used)), reverse=True), (p for p in range(len(used)) if p not in used)))
    for a, b in moves:
        pool[:, b] = pool[:, a]
    now = dict(moves)
    after = [[now.get(p, p) for p in row[:n]] + row[n:] for row, n in zip(table, pages)]
    pad = [-1] * (n_pages // 2 + 1 - len(moves))
    return [torch.tensor(t, dtype=torch.int32) for t in (after, [a for a, _ in moves] + pad, [b for _, b in moves] + pad, [len(used), len(moves), len(used)])] + [pool]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] in ("sample", "filter"):
        rows = case["rows"] if case["kind"] == "sample" else case["batch"] * (case["k"] + 1)
        n = rows * case["vocab"]
        return {"bytes": int(n * (2 if case["dtype"] == "bf16" else 4) * (1 if case["kind"] == "sample" else 2)), "flops": int(4 * n)}
    if case["kind"] == "fork":
        n = case["sources"] * case["copies"]
        entries = n * case["kv"] * 0.75 / PAGE
        return {"bytes": int(n * 15 / 16 * 2 * case["layers"] * case["page"] + 8 * entries + 28 * n), "flops": int(n)}
    entries = case["batch"] * (case["kv"] * 0.625 / PAGE + 0.5)
    n_pages = entries / (1 - case["spare"])
    if case["kind"] == "free":
        return {"bytes": int(4 * (entries + n_pages)), "flops": int(entries)}
    used = entries * (1 - case["shared"] * 7 / 8 * 0.6)
    moves = used * max(0.0, 1 - used / n_pages)
    return {"bytes": int(moves * 2 * case["layers"] * case["page"] + 8 * entries + 4 * n_pages), "flops": int(entries)}

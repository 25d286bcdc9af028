"""Timed cases of the serving operators: prompts of different lengths, the paged cache, and its pages.

Four kinds.  ``prompt``: attention over packed prompts of different lengths.  ``append``: new K/V
rows into a paged cache, one token a sequence or whole packed prompts.  ``decode``: the new token's
n positions against the paged cache.  ``pages``: who holds which page (free, fork, grow, compact)
and the page copies that follow from it.

``run`` computes the plain form in elementary torch operations in 32 bits, or, with ``own`` true,
makes the calls of ``paper_2607_08186_gb300.binding``.  Head layouts and lengths are the ones the
repository's own configurations, tests and benchmark use.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
MODES = {"within": 0, "cross": 1, "local": 2}

# (query heads, K/V heads, head dim): 8B-class dense, large-MoE-class, 617B grouping, 80B, and small heads
HEADS = [(32, 8, 128), (64, 8, 128), (96, 8, 128), (24, 2, 256), (16, 4, 64), (4, 4, 64)]
MAX_CACHE_BYTES = 4.0e9     # a drawn cache, below the largest listed one
MAX_SCORES = 6.0e9          # a drawn prompt's query-key pairs in the plain form, below the largest listed one
MAX_POOL_BYTES = 5.0e8      # one pool of a drawn page case


def _attn(name, kind, mode, lens, n, heads, P=0, window=0, pad=0):
    """lens: "longest x count", spread by _spread; P: tokens a page; pad: tokens behind the last sequence."""
    return {"name": name, "kind": kind, "mode": mode, "L": lens[0], "B": lens[1], "n": n, "Hq": heads[0], "Hkv": heads[1],
            "Dh": heads[2], "P": P, "window": window, "pad": pad, "idle": 0}


def _pages(name, what, pages, B, P, n, heads, forks=0):
    return {"name": name, "kind": "pages", "what": what, "pages": pages, "B": B, "P": P, "n": n, "Hkv": heads[1],
            "Dh": heads[2], "forks": forks}


def listed():
    return [
        # smallest: two short sequences of the tiny configuration: launches and latency
        _attn("decode_tiny", "decode", "within", (64, 2), 2, (4, 4, 64), P=8),
        # single-user decoding at 8k tokens: one intra-stream layer's step
        _attn("decode_8b_b1_8k", "decode", "within", (8192, 1), 4, (32, 8, 128), P=16),
        # a serving batch of 16 sequences of different lengths up to 32k tokens, cross-stream layer (the most bytes)
        _attn("decode_8b_b16_32k", "decode", "cross", (32768, 16), 4, (32, 8, 128), P=32),
        # a small serving batch of the 80B configuration (head dim 256)
        _attn("decode_80b_b4_8k", "decode", "within", (8192, 4), 4, (24, 2, 256), P=16),
        # the new token of each of 64 running sequences into the cache
        _attn("append_tokens_8b_b64", "append", "token", (2048, 64), 4, (32, 8, 128), P=16),
        # a batch of prompts into the cache after their prefill
        _attn("append_prompts_8b", "append", "prompt", (4000, 6), 4, (32, 8, 128), P=16, pad=37),
        # requests finish, others start from live prefixes: a small pool
        _pages("pages_turnover_small", "turnover", 300, 12, 8, 2, (4, 4, 64), forks=3),
        # the same on an 8B-class layer's pools: 64 slots, 24 requests that share prefixes
        _pages("pages_turnover_8b", "turnover", 4096, 64, 16, 4, (32, 8, 128), forks=24),
        # a pool with holes drawn together, and the layer's pages moved
        _pages("pages_compact_8b", "compact", 4096, 64, 16, 4, (32, 8, 128)),
        # many short prompts of a small model: head dim 64, odd stream count, lengths off every tile size
        _attn("prompt_dh64_b24", "prompt", "within", (701, 24), 3, (16, 4, 64), pad=5),
        # prompts of an 8B-class cross-stream layer (the most arithmetic)
        _attn("prompt_8b_cross", "prompt", "cross", (1801, 4), 4, (32, 8, 128)),
        # prompts of an 80B-class intra-stream layer
        _attn("prompt_80b_within", "prompt", "within", (1533, 5), 4, (24, 2, 256), pad=100),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "append", "pages", "prompt", "prompt"])
    n = rng.choice([1, 2, 3, 4, 4, 8])
    heads = rng.choice(HEADS)
    P = rng.choice([1, 3, 8, 16, 16, 20, 32, 64])
    if kind == "pages":
        B = _log_int(rng, 2, 200)
        c = _pages("", rng.choice(["turnover", "turnover", "compact"]), _log_int(rng, 4 * B, 20000), B, P, n, heads,
                   forks=rng.randint(1, max(1, B // 3)))
        while c["pages"] * P * n * heads[1] * heads[2] * 2.0 > MAX_POOL_BYTES and c["pages"] > 4 * B:
            c["pages"] = max(4 * B, c["pages"] * 3 // 4)
        while c["pages"] * c["P"] * n * heads[1] * heads[2] * 2.0 > MAX_POOL_BYTES:
            c["P"] = max(1, c["P"] // 2)
        del c["name"]
        return c
    mode = rng.choice(["within", "cross", "local"])
    if kind == "decode":
        c = _attn("", kind, mode, (_log_int(rng, 1, 32768), rng.choice([1, 2, 4, 7, 16, 33])), n, heads, P)
        c["idle"] = rng.choice([0, 0, 1]) if c["B"] > 1 else 0
        while 4.0 * c["B"] * c["L"] * n * heads[1] * heads[2] > MAX_CACHE_BYTES:
            c["L"] = c["L"] * 3 // 4
    elif kind == "append":
        what = rng.choice(["token", "prompt"])
        c = _attn("", kind, what, (_log_int(rng, 1, 4096), _log_int(rng, 1, 64)), n, heads, P,
                  pad=rng.choice([0, 1, 50]) if what == "prompt" else 0)
        c["idle"] = rng.choice([0, 0, 1]) if c["B"] > 1 else 0
        while c["B"] * c["L"] * n * heads[1] * heads[2] * 2.0 > 2 * MAX_POOL_BYTES:
            c["L"] = max(1, c["L"] * 3 // 4)
    else:
        c = _attn("", kind, mode, (_log_int(rng, 1, 4096), _log_int(rng, 1, 40)), n, heads, pad=rng.choice([0, 0, 1, 130]))
        c["idle"] = rng.choice([0, 0, 1]) if c["B"] > 1 else 0
        while _plain_scores(c) > MAX_SCORES:
            c["L"] = max(1, c["L"] * 3 // 4)
            c["B"] = c["B"] if c["L"] > 8 else max(1, c["B"] // 2)
    if mode == "local" and kind != "append":
        c["window"] = _log_int(rng, 1, 4096)
    del c["name"]
    return c


# ------------------------------------------------------------------ state

class State:
    pass


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 7919 + 17)


def _randn(g, *shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, 1.0, generator=g)


def _spread(c):
    """Tokens of each sequence: the first has L, the others a quarter of it to all of it (prompts: a hundredth
    to all of it); `idle` more of them hold nothing."""
    low = 0.01 if c["kind"] == "prompt" or c["mode"] == "prompt" else 0.25
    lens = [c["L"]] + [max(1, int(c["L"] * (low + (1 - low) * (0.6180339887 * b % 1.0)))) for b in range(1, c["B"])]
    for b in range(c["idle"]):
        lens[-1 - b] = 0
    return lens


def _plain_scores(c):
    N = sum(_spread(c)) + c["pad"]
    return float(N) * N * c["Hq"] * c["n"] * (1 if c["mode"] == "within" else c["n"])


def _offsets(counts):
    off = [0]
    for x in counts:
        off.append(off[-1] + x)
    return off


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _table(g, lens, P, pages):
    """Pages of the sequences in random order over the pool; entries that hold nothing are -1."""
    held = [-(-x // P) for x in lens]
    width = max(1, max(held))
    at = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    perm = torch.randperm(pages, generator=g, device=DEV).int()
    mask = torch.arange(width, device=DEV)[None] < _int(held)[:, None]
    at[mask] = perm[:sum(held)]
    return at


def _pool_sizes(c):
    """Slots of a page case: tokens held by each.  The last `forks` slots hold requests that have finished."""
    B, P = c["B"], c["P"]
    most = max(1, int(c["pages"] * 0.55 / B)) * P  # a bit over half of the pool is held
    return [max(1, int(most * (0.3 + 0.7 * (0.6180339887 * (b + 1) % 1.0)))) for b in range(B)]


def prepare(case, seed):
    s, g = State(), _gen(seed)
    s.case = c = dict(case)
    s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
    s.ws = None
    n, Hkv, Dh, B, P = c["n"], c["Hkv"], c["Dh"], c["B"], c["P"]
    if c["kind"] == "pages":
        lens = _pool_sizes(c)
        s.lens = _int(lens)
        s.table = torch.full((B, max(1, c["pages"] // B + 2)), -1, dtype=torch.int32, device=DEV)
        t = _table(g, lens, P, c["pages"])
        s.table[:, :t.shape[1]] = t
        s.refs = torch.zeros(c["pages"], dtype=torch.int32, device=DEV)
        s.refs[t[t >= 0].long()] = 1
        s.k, s.v = _randn(g, c["pages"], P * n, Hkv, Dh), _randn(g, c["pages"], P * n, Hkv, Dh)
        if c["what"] == "turnover":
            F = min(c["forks"], B - 1)
            live = B - F
            src = [i % live for i in range(F)]
            s.dst, s.src = _int(list(range(live, B))), _int(src)
            # each new request shares a prefix that ends anywhere in a page, and brings tokens of its own
            share = (torch.rand(F, generator=g, device=DEV) * s.lens[s.src.long()]).int()
            s.tokens = share
            s.add = torch.zeros(B, dtype=torch.int32, device=DEV)
            s.add[live:] = (torch.rand(F, generator=g, device=DEV) * 0.4 * min(lens)).int() + 1
            s.copies = torch.full((F, 2), -1, dtype=torch.int32, device=DEV)
        else:
            s.moves = torch.full((max(1, c["pages"] // 2), 2), -1, dtype=torch.int32, device=DEV)
            s.new_refs, s.new_table = torch.empty_like(s.refs), torch.empty_like(s.table)
        return s
    Hq, lens = c["Hq"], _spread(c)
    if c["kind"] == "prompt":
        N = sum(lens) + c["pad"]
        s.offsets = _int(_offsets(lens))
        s.q, s.k, s.v = _randn(g, N * n, Hq, Dh), _randn(g, N * n, Hkv, Dh), _randn(g, N * n, Hkv, Dh)
        s.o = torch.zeros_like(s.q)
        s.lse = torch.zeros(Hq, N * n, dtype=torch.float32, device=DEV)
        return s
    held = [-(-x // P) for x in lens]
    pages = sum(held) + max(1, sum(held) // 16)
    s.table, s.lens = _table(g, lens, P, pages), _int(lens)
    s.k, s.v = _randn(g, pages, P * n, Hkv, Dh), _randn(g, pages, P * n, Hkv, Dh)
    if c["kind"] == "append":
        if c["mode"] == "token":
            s.offsets = None
            s.kn, s.vn = _randn(g, B, n, Hkv, Dh), _randn(g, B, n, Hkv, Dh)
        else:  # the last tokens of each sequence are new: all of the even ones', half of the others'
            new = [x if b % 2 == 0 else x // 2 for b, x in enumerate(lens)]
            N = sum(new) + c["pad"]
            s.offsets = _int(_offsets(new))
            s.kn, s.vn = _randn(g, max(1, N) * n, Hkv, Dh), _randn(g, max(1, N) * n, Hkv, Dh)
        return s
    s.q = _randn(g, B, n, Hq, Dh)
    s.o = torch.empty_like(s.q)
    s.lse = torch.empty(B, Hq, n, dtype=torch.float32, device=DEV)
    return s


def run(s):
    return {"decode": _decode, "append": _append, "prompt": _prompt, "pages": _pages_pass}[s.case["kind"]](s)


# ------------------------------------------------------------------ the framework's calls

def _workspace(s, nbytes):
    if s.ws is None:
        s.ws = torch.empty(max(1, nbytes), dtype=torch.uint8, device=DEV)
    return s.ws


def _decode(s):
    if not own:
        return _plain_decode(s)
    from paper_2607_08186_gb300 import binding as hd
    c = s.case
    if s.ws is None:
        _workspace(s, hd.sfa_decode_paged_workspace_bytes(c["B"], c["L"], c["n"], c["Hq"], c["Hkv"], c["Dh"],
                                                          MODES[c["mode"]], c["window"]))
    hd.sfa_decode_paged(s.q, s.k, s.v, s.table, s.lens, s.o, c["n"], MODES[c["mode"]], s.ws, max_tokens=c["L"], lse=s.lse,
                        window=c["window"], dev_status=s.status)
    return {"o": s.o, "lse": s.lse, "status": s.status}


def _append(s):
    if not own:
        return _plain_append(s)
    from paper_2607_08186_gb300 import binding as hd
    hd.sfa_kv_append_paged(s.kn, s.vn, s.k, s.v, s.table, s.lens, s.case["n"], offsets=s.offsets, dev_status=s.status)
    return {"k": s.k, "v": s.v, "status": s.status}


def _prompt(s):
    if not own:
        return _plain_prompt(s)
    from paper_2607_08186_gb300 import binding as hd
    c = s.case
    if s.ws is None:
        _workspace(s, hd.sfa_fwd_packed_workspace_bytes(c["B"], s.q.shape[0] // c["n"], c["n"], c["Hq"], c["Hkv"], c["Dh"],
                                                        MODES[c["mode"]]))
    hd.sfa_fwd_packed(s.q, s.k, s.v, s.o, s.lse, s.offsets, c["n"], MODES[c["mode"]], s.ws, window=c["window"],
                      dev_status=s.status)
    return {"o": s.o, "lse": s.lse, "status": s.status}


def _pages_pass(s):
    """turnover: finished requests give their pages back, new ones fork live prefixes into the same slots (the
    last, partly filled page of a prefix is copied) and get pages for their own tokens.  A second pass over the
    same state frees what the first one made and makes it again.  compact: tables and counts of the drawn-together
    pool beside the old ones, and the moves' pages copied (into pages nobody holds)."""
    if not own:
        return _plain_turnover(s) if s.case["what"] == "turnover" else _plain_compact(s)
    from paper_2607_08186_gb300 import binding as hd
    c = s.case
    ws = s.ws if s.ws is not None else _workspace(s, hd.hd_pages_workspace_bytes(c["B"], c["pages"]))
    if c["what"] == "turnover":
        hd.hd_pages_free(s.refs, s.table, s.lens, s.dst, c["P"], dev_status=s.status)
        hd.hd_pages_fork(s.refs, s.table, s.lens, s.src, s.dst, s.tokens, s.copies, c["P"], ws, dev_status=s.status)
        hd.hd_pages_copy(s.k, s.v, s.copies, dev_status=s.status)
        hd.hd_pages_grow(s.refs, s.table, s.lens, s.add, c["P"], ws, dev_status=s.status)
        return {"refs": s.refs, "table": s.table, "lens": s.lens, "copies": s.copies, "k": s.k, "v": s.v, "status": s.status}
    hd.hd_pages_compact(s.refs, s.table, s.lens, s.new_refs, s.new_table, s.moves, c["P"], ws, dev_status=s.status)
    hd.hd_pages_copy(s.k, s.v, s.moves, dev_status=s.status)
    return {"refs": s.new_refs, "table": s.new_table, "moves": s.moves, "k": s.k, "v": s.v, "status": s.status}


# ------------------------------------------------------------------ plain forms

def _softmax_rows(z, v):
    """(P v, lse) of scores z with -inf where nothing is seen; rows that see nothing give 0 and -inf.  z is used up."""
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = z.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(l > 0, l, torch.ones_like(l))
    return o, (m + torch.log(l)).squeeze(-1)


def _plain_decode(s):
    c = s.case
    B, n, Hq, Hkv, Dh, P = (c[x] for x in ("B", "n", "Hq", "Hkv", "Dh", "P"))
    G, width = Hq // Hkv, s.table.shape[1]
    at = s.table.clamp(min=0).long()
    k = s.k[at].view(B, width * P * n, Hkv, Dh).permute(0, 2, 3, 1).float()
    v = s.v[at].view(B, width * P * n, Hkv, Dh).permute(0, 2, 1, 3).float()
    q = s.q.float().view(B, n, Hkv, G, Dh).transpose(1, 2).reshape(B, Hkv, n * G, Dh)
    z = torch.matmul(q, k).mul_(1.0 / math.sqrt(Dh)).view(B, Hkv, n, G, -1)
    kp = torch.arange(width * P * n, device=DEV)
    qp = (s.lens.long()[:, None] - 1) * n + torch.arange(n, device=DEV)  # [B][n]
    see = kp <= qp[..., None]
    if c["mode"] == "within":
        see &= kp % n == torch.arange(n, device=DEV)[:, None]
    if c["mode"] == "local":
        see &= kp > qp[..., None] - c["window"]
    see &= (s.lens > 0)[:, None, None]
    z.masked_fill_(~see[:, None, :, None], -math.inf)
    o, lse = _softmax_rows(z.view(B, Hkv, n * G, -1), v)
    o = o.view(B, Hkv, n, G, Dh).transpose(1, 2).reshape(B, n, Hq, Dh).to(torch.bfloat16)
    return {"o": o, "lse": lse.view(B, Hkv, n, G).transpose(2, 3).reshape(B, Hq, n), "status": s.status}


def _plain_append(s):
    c = s.case
    n, P, Hkv, Dh = c["n"], c["P"], c["Hkv"], c["Dh"]
    lens = s.lens.long()
    if s.offsets is None:
        b = torch.arange(c["B"], device=DEV)
        t, use = lens - 1, lens > 0
    else:
        off = s.offsets.long()
        i = torch.arange(s.kn.shape[0] // n, device=DEV)
        b = (torch.searchsorted(off, i, right=True) - 1).clamp(0, c["B"] - 1)
        use = (i >= off[0]) & (i < off[-1])
        t = lens[b] - off[b + 1] + i
    t = t.clamp(min=0)
    row = s.table[b, t // P].long() * P + t % P
    s.k.view(-1, n, Hkv, Dh)[row[use]] = s.kn.view(-1, n, Hkv, Dh)[use]
    s.v.view(-1, n, Hkv, Dh)[row[use]] = s.vn.view(-1, n, Hkv, Dh)[use]
    return {"k": s.k, "v": s.v, "status": s.status}


def _plain_prompt(s):
    c = s.case
    n, Hq, Hkv, Dh, w = c["n"], c["Hq"], c["Hkv"], c["Dh"], c["window"]
    G, N = Hq // Hkv, s.q.shape[0] // n
    within = c["mode"] == "within"
    R = n if within else 1          # separate problems, of M rows each
    M = N if within else N * n
    off = s.offsets.long()
    token = torch.arange(N, device=DEV)
    seq = torch.searchsorted(off, token, right=True)
    real = (token >= off[0]) & (token < off[-1])
    if not within:
        seq, real = seq.repeat_interleave(n), real.repeat_interleave(n)
    at = torch.arange(M, device=DEV)
    see = (seq[:, None] == seq) & (at <= at[:, None]) & real[:, None] & real
    if c["mode"] == "local":
        see &= at > at[:, None] - w
    q = s.q.view(M, R, Hkv, G, Dh).permute(1, 2, 3, 0, 4).reshape(R, Hkv, G * M, Dh).float()
    k = s.k.view(M, R, Hkv, Dh).permute(1, 2, 3, 0).float()
    v = s.v.view(M, R, Hkv, Dh).permute(1, 2, 0, 3).float()
    z = torch.matmul(q, k).mul_(1.0 / math.sqrt(Dh)).view(R, Hkv, G, M, M)
    z.masked_fill_(~see, -math.inf)
    o, lse = _softmax_rows(z.view(R, Hkv, G * M, M), v)
    o = o.view(R, Hkv, G, M, Dh).permute(3, 0, 1, 2, 4).reshape(M, R, Hq, Dh)
    lse = lse.view(R, Hq, M).permute(1, 2, 0).reshape(Hq, M, R)
    keep = real.view(M, 1, 1, 1)
    o = torch.where(keep, o.to(torch.bfloat16), s.o.view(M, R, Hq, Dh)).reshape(N * n, Hq, Dh)
    lse = torch.where(real.view(1, M, 1), lse, s.lse.view(Hq, M, R)).reshape(Hq, N * n)
    return {"o": o, "lse": lse, "status": s.status}


def _free_ids(refs):
    """Ids of the free pages first, ascending; and how many there are."""
    return torch.sort((refs > 0).to(torch.int8), stable=True)[1].int(), (refs == 0).sum()


def _plain_turnover(s):
    c = s.case
    P, width = c["P"], s.table.shape[1]
    refs, table, lens = s.refs, s.table, s.lens
    i = torch.arange(width, device=DEV)
    dst, src = s.dst.long(), s.src.long()
    one = torch.ones((), dtype=torch.int32, device=DEV)
    none = torch.full((), -1, dtype=torch.int32, device=DEV)
    # free
    held = i < ((lens[dst] + P - 1) // P)[:, None]
    refs.index_add_(0, table[dst].clamp(min=0).long().flatten(), torch.where(held, -one, 0 * one).flatten())
    table[dst] = none
    lens[dst] = 0
    # fork
    ids, avail = _free_ids(refs)
    part = (s.tokens % P > 0)
    rank = torch.cumsum(part, 0) - 1
    ok = ~part | (rank < avail)
    full = s.tokens // P
    fresh = ids[rank.clamp(0, len(ids) - 1)]
    take = part & ok
    shared = (i < full[:, None]) & ok[:, None]
    rows = torch.where(shared, table[src], none)
    last = (i == full[:, None]) & take[:, None]
    refs.index_add_(0, rows.clamp(min=0).long().flatten(), torch.where(shared, one, 0 * one).flatten())
    refs.index_add_(0, fresh.long(), take.int())
    old = table[src, full.clamp(max=width - 1).long()]
    table[dst] = torch.where(last, fresh[:, None], rows)
    lens[dst] = torch.where(ok, s.tokens, 0 * s.tokens)
    s.copies.copy_(torch.where(take[:, None], torch.stack([old, fresh], 1), none))
    # copy
    _copy_pages(s, s.copies)
    # grow
    ids, avail = _free_ids(refs)
    have, want = (lens + P - 1) // P, (lens + s.add + P - 1) // P
    need = want - have
    upto = torch.cumsum(need, 0)
    ok = (need == 0) | (upto <= avail)
    base = upto - need
    new = (i >= have[:, None]) & (i < want[:, None]) & ok[:, None]
    which = (base[:, None] + i - have[:, None]).clamp(0, len(ids) - 1)
    got = ids[which.long()]
    refs.index_add_(0, got.long().flatten(), new.int().flatten())
    table.copy_(torch.where(new, got, table))
    lens.copy_(torch.where(ok, lens + s.add, lens))
    return {"refs": refs, "table": table, "lens": lens, "copies": s.copies, "k": s.k, "v": s.v, "status": s.status}


def _copy_pages(s, pairs):
    """Page a onto page b in both pools for the pairs (a, b); pairs of -1 are left out."""
    a, b = pairs[pairs[:, 0] >= 0].long().T
    s.k[b] = s.k[a]
    s.v[b] = s.v[a]


def _plain_compact(s):
    P, pages = s.case["P"], s.refs.shape[0]
    live = s.refs > 0
    K = live.sum()
    at = torch.arange(pages, device=DEV)
    high, low = live & (at >= K), ~live & (at < K)
    ids_high = torch.sort((~high).to(torch.int8), stable=True)[1]
    ids_low = torch.sort((~low).to(torch.int8), stable=True)[1]
    M = s.moves.shape[0]
    some = at[:M] < high.sum()
    moves = torch.where(some[:, None], torch.stack([ids_high[:M], ids_low[:M]], 1), torch.full((), -1, device=DEV))
    s.moves.copy_(moves)
    to = torch.cat([at, at[:1]])
    to.index_copy_(0, torch.where(some, moves[:, 0], torch.full_like(moves[:, 0], pages)), moves[:, 1])
    to = to[:-1]
    s.new_refs.zero_().index_add_(0, to, torch.where(live, s.refs, torch.zeros_like(s.refs)))
    held = torch.arange(s.table.shape[1], device=DEV) < ((s.lens + P - 1) // P)[:, None]
    s.new_table.copy_(torch.where(held, to[s.table.clamp(min=0).long()].int(), torch.full_like(s.table, -1)))
    _copy_pages(s, s.moves)
    return {"refs": s.new_refs, "table": s.new_table, "moves": s.moves, "k": s.k, "v": s.v, "status": s.status}


# ------------------------------------------------------------------ work

def _pairs(c, T, first):
    """Visible (query, key) pairs of one query head over positions first .. T*n - 1 of a sequence of T tokens."""
    n, w = c["n"], c["window"]
    if c["mode"] == "within":
        a, b = first // n, T
        return n * (b * (b + 1) - a * (a + 1)) // 2

    def upto(p):  # sum of min(q + 1, w) for q < p
        m = p if c["mode"] == "cross" else min(w, p)
        return m * (m + 1) // 2 + (p - m) * m

    return upto(T * n) - upto(first)


def work(case):
    c = case
    n, Hkv, Dh, P = c["n"], c["Hkv"], c["Dh"], c["P"]
    if c["kind"] == "pages":
        page = 4 * P * n * Hkv * Dh  # one page of both pools
        lens = _pool_sizes(c)
        held = [-(-x // P) for x in lens]
        if c["what"] == "turnover":
            F = min(c["forks"], c["B"] - 1)
            # about one page in P needs no copy; tables of the slots that change, reference counts once
            return {"bytes": 2.0 * page * F * (1 - 1 / P) + 4.0 * c["pages"] + 8.0 * sum(held[-F:]) + 24.0 * F, "flops": 0.0}
        K = sum(held)
        moves = K * (c["pages"] - K) / c["pages"]  # live pages beyond the first K, on average
        return {"bytes": 2.0 * page * moves + 8.0 * c["pages"] + 8.0 * K + 8.0 * moves, "flops": 0.0}
    lens = _spread(c)
    if c["kind"] == "append":
        rows = sum(x > 0 for x in lens) if c["mode"] == "token" else sum(x if b % 2 == 0 else x // 2 for b, x in enumerate(lens))
        return {"bytes": 8.0 * rows * n * Hkv * Dh + 8.0 * c["B"], "flops": 0.0}
    Hq = c["Hq"]
    if c["kind"] == "decode":
        keys = sum(min(n * T, c["window"] + n - 1) if c["mode"] == "local" else n * T for T in lens)
        pairs = sum(_pairs(c, T, (T - 1) * n) for T in lens if T)
        return {"bytes": float(keys * Hkv * Dh * 4 + c["B"] * (4 * n * Hq * Dh + 4 * n * Hq) + 4 * keys // (n * P)),
                "flops": 4.0 * Dh * Hq * pairs}
    rows = n * sum(lens)
    pairs = sum(_pairs(c, T, 0) for T in lens)
    return {"bytes": float(rows * (4 * Hq * Dh + 4 * Hkv * Dh + 4 * Hq)), "flops": 4.0 * Dh * Hq * pairs}


# ------------------------------------------------------------------ 64-bit reference

def _exact_rows(c, q, k, v, first, o, lse):
    """One sequence: q [rows][Hq][Dh] at positions first ..., k, v [positions][Hkv][Dh]; o, lse [Hq][rows] written."""
    n, G, Dh = c["n"], c["Hq"] // c["Hkv"], c["Dh"]
    kp = torch.arange(k.shape[0], device=DEV)
    for h in range(c["Hq"]):
        kh, vh = k[:, h // G].double(), v[:, h // G].double()
        for a in range(0, q.shape[0], 4096):
            qp = first + torch.arange(a, min(a + 4096, q.shape[0]), device=DEV)
            z = q[a:a + 4096, h].double() @ kh.T / math.sqrt(Dh)
            vis = kp[None] <= qp[:, None]
            if c["mode"] == "within":
                vis &= (kp[None] - qp[:, None]) % n == 0
            elif c["mode"] == "local":
                vis &= qp[:, None] - kp[None] < c["window"]
            z[~vis] = -math.inf
            e = torch.logsumexp(z, 1)
            o[a:a + 4096, h] = torch.exp(z - e[:, None]) @ vh
            lse[h, a:a + 4096] = e


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    n, P = c["n"], c["P"]
    f64 = dict(dtype=torch.float64, device=DEV)
    if c["kind"] == "decode":
        o, lse = torch.zeros(s.q.shape, **f64), torch.full(s.lse.shape, -math.inf, **f64)
        for b, T in enumerate(_spread(c)):
            if T:
                ids = s.table[b, :-(-T // P)].long()
                k, v = (x[ids].flatten(0, 1)[:T * n] for x in (s.k, s.v))
                _exact_rows(c, s.q[b], k, v, (T - 1) * n, o[b], lse[b])
        return {"o": o, "lse": lse, "status": s.status}
    if c["kind"] == "prompt":
        o, lse = s.o.double(), s.lse.double()
        at = 0
        for T in _spread(c):
            r = slice(at * n, (at + T) * n)
            if T:
                _exact_rows(c, s.q[r], s.k[r], s.v[r], 0, o[r], lse[:, r])
            at += T
        return {"o": o, "lse": lse, "status": s.status}
    if c["kind"] == "append":
        table, lens = s.table.tolist(), _spread(c)
        off = s.offsets.tolist() if s.offsets is not None else None
        dst, src = [], []
        for b, T in enumerate(lens):
            new = min(1, T) if off is None else off[b + 1] - off[b]
            for i in range(new):
                t = T - new + i
                dst.append(table[b][t // P] * P + t % P)
                src.append(b if off is None else off[b] + i)
        for pool, rows in ((s.k, s.kn), (s.v, s.vn)):
            if dst:
                pool.view(-1, n, c["Hkv"], c["Dh"])[torch.tensor(dst, device=DEV)] = \
                    rows.view(-1, n, c["Hkv"], c["Dh"])[torch.tensor(src, device=DEV)]
        return {"k": s.k, "v": s.v, "status": s.status}
    refs, table, lens = s.refs.tolist(), s.table.tolist(), s.lens.tolist()
    if c["what"] == "turnover":
        for b in s.dst.tolist():
            for i in range(-(-lens[b] // P)):
                refs[table[b][i]] -= 1
                table[b][i] = -1
            lens[b] = 0
        copies = []
        for a, b, t in zip(s.src.tolist(), s.dst.tolist(), s.tokens.tolist()):
            pair = [-1, -1]
            if t % P:
                if 0 not in refs:
                    copies.append(pair)
                    continue
                new = refs.index(0)
                refs[new] = 1
                pair = [table[a][t // P], new]
                table[b][t // P] = new
            for i in range(t // P):
                table[b][i] = table[a][i]
                refs[table[a][i]] += 1
            lens[b] = t
            copies.append(pair)
        pairs = copies
        left, used = refs.count(0), 0
        for b, x in enumerate(s.add.tolist()):
            have, want = -(-lens[b] // P), -(-(lens[b] + x) // P)
            used += want - have
            if want == have or used <= left:
                lens[b] += x
                for i in range(have, want):
                    table[b][i] = refs.index(0)
                    refs[table[b][i]] = 1
        got = {"refs": _int(refs), "table": _int(table), "lens": _int(lens), "copies": _int(copies)}
    else:
        live = [p for p, r in enumerate(refs) if r]
        K = len(live)
        pairs = list(map(list, zip([p for p in live if p >= K], [p for p in range(K) if not refs[p]])))
        to = dict(map(tuple, pairs))
        new = [0] * len(refs)
        for p in live:
            new[to.get(p, p)] = refs[p]
        rows = [[to.get(p, p) if i < -(-lens[b] // P) else -1 for i, p in enumerate(row)] for b, row in enumerate(table)]
        moves = (pairs + [[-1, -1]] * s.moves.shape[0])[:s.moves.shape[0]]
        got = {"refs": _int(new), "table": _int(rows), "moves": _int(moves)}
    pairs = [p for p in pairs if p[0] >= 0]
    if pairs:
        a, b = torch.tensor(pairs, device=DEV).T
        for pool in (s.k, s.v):
            pool[b] = pool[a]
    return {**got, "k": s.k, "v": s.v, "status": s.status}

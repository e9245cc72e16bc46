"""More operators on a paged cache, measured: what a serving program does from the prompt on with a cache that is kept short.

  attention  of the new rows of every sequence (a prompt, a few drafted tokens, a single token) over the rows of its pages up to
             each one's own place, within a sliding window and among the first rows (sinks), with the rows' log-sum-exp
  weights    the attention weights that these rows give to every cached row, summed over queries and query heads into a weight
             per row that is kept beside the pages
  evict      of every head the rows with the largest accumulated weight beside the first and the newest ones, moved in order
             into fresh pages, with their weights and the pages' key bounds

A page holds `page` rows of one KV head; a head's pages come from a table [batch, hkv, pages]; heads of one sequence may have
different lengths.  4-bit rows: 32 neighbouring elements share a step S and a base B, both fp16, and an element is
B + S (1 + code / 16).  Row t of a head's `new` ones has the place length - new + t; it sees the places j <= place with
j > place - window or j < first.

A case is a dict of plain values.  `own` False: elementary torch operations; True: the library's entry points.
"""
import math

import torch

own = False

DEV = "cuda:0"
ALL = 2 ** 30                # a window that no row is outside of
BLOCK = 2 ** 30              # scores of a block of queries in the plain form


# ------------------------------------------------------------------------------------------------- the cases
def _case(op, **kw):
    """lo, hi: rows of the shortest and the longest sequence (or head, with per_head), the new ones among them; new: rows of
    queries per head, 0: all rows; pad: rows of queries behind the last sequence; window, first: what a row sees; keep: rows that
    are kept of the longest head, shorter heads in proportion; last: newest rows kept whatever their weight."""
    c = dict(op=op, fmt="rows", dtype="bf16", batch=1, hq=28, hkv=4, d=128, page=64, lo=8192, hi=8192, per_head=False, new=1,
             pad=0, window=ALL, first=0, keep=0, last=0, bounds=False)
    c.update(kw)
    return c


def listed():
    return [
        # the new token of one sequence, a window of a thousand rows behind four sinks: latency
        _case("attention", name="attention_step_one", lo=8193, hi=8193, window=1024, first=4),
        # a decoding step of 64 sequences of 1 to 16384 tokens on 4-bit pages, a window of 4096 rows
        _case("attention", name="attention_step_batch_4bit", fmt="4bit", batch=64, hq=32, hkv=8, lo=1, hi=16384, window=4096, first=64),
        # five drafted tokens of 16 sequences to be verified, no window
        _case("attention", name="attention_draft", batch=16, hq=32, hkv=8, lo=3000, hi=32768, new=5),
        # two prompts of 5 to 16 thousand tokens, causal, in a batch padded at its end
        _case("attention", name="attention_prompts", batch=2, lo=5001, hi=16384, new=0, pad=77),
        # a prompt of 32 thousand tokens on 4-bit pages, within a window
        _case("attention", name="attention_prompt_window_4bit", fmt="4bit", lo=32768, hi=32768, new=0, window=4096, first=16),
        # the next hundred rows of two fp32 caches of a small model, heads of unequal length
        _case("attention", name="attention_chunk_f32", dtype="f32", batch=2, hq=16, hkv=8, d=64, page=32, lo=133, hi=2000, per_head=True,
              new=100, window=700, first=3),
        # a decoding step's weights of one sequence on 4-bit pages: latency
        _case("weights", name="weights_step_one_4bit", fmt="4bit", lo=4097, hi=4097),
        # a decoding step's weights of 32 sequences
        _case("weights", name="weights_step_batch", batch=32, hq=32, hkv=8, lo=1, hi=16384),
        # the weights that two prompts give to their own rows, within a window
        _case("weights", name="weights_prompts", batch=2, lo=4000, hi=16384, new=0, window=8192, first=16, pad=5),
        # one sequence that has grown by 64 tokens over its budget: latency
        _case("evict", name="evict_step_one", lo=2112, hi=2112, keep=2048, first=4, last=64),
        # 32 sequences on 4-bit pages to half their length, and what is left read back
        _case("evict", name="evict_batch_4bit", fmt="4bit", batch=32, hq=32, hkv=8, page=32, lo=2000, hi=16384, keep=8192, first=16, last=256, bounds=True),
        # heads of up to 131072 rows to an eighth
        _case("evict", name="evict_long", batch=2, lo=60000, hi=131072, per_head=True, keep=16384, first=4, last=1024, bounds=True),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def _cost(c):
    """Seconds, roughly, of a kernel; and of the plain form, that takes every row for every query."""
    w = work(c)
    elements = c["batch"] * c["hq"] * max(_counts(c)) * c["hi"] if c["op"] != "evict" else 0
    rate = 1.0e14 if c["dtype"] == "f32" else 1.0e15
    return max(w["bytes"] / 5e12, w["flops"] / rate), elements


def draw(rng):
    """One more case of the same ranges: one to 64 sequences of one to 131072 rows, both formats and types, one new row to
    whole prompts, windows of one row to all of them."""
    op = rng.choice(["attention", "attention", "attention", "weights", "weights", "evict"])
    most = [_cost(c) for c in listed() if c["op"] == op]
    most = [max(x) for x in zip(*most)]
    hq, hkv = rng.choice([(28, 4), (32, 8), (16, 8), (12, 2), (4, 2), (40, 8), (8, 8), (32, 2)])
    d = rng.choice([128, 128, 64])
    fmt, dtype = rng.choice([("4bit", "bf16")] * 2 + [("rows", "bf16")] * 3 + [("rows", "f32")])
    c = _case(op, fmt=fmt, dtype=dtype, batch=_log(rng, 1, 64), hq=hq, hkv=hkv, d=d, page=rng.choice([32, 64, 64, 128]), hi=_log(rng, 2, 131072),
              per_head=rng.random() < 0.3, pad=rng.choice([0, 0, 5, 64]))
    share, some, wide, far = rng.random(), _log(rng, 1, 300), rng.random(), rng.random()
    kind = rng.choice(["one", "one", "some", "some", "all"])
    c["first"] = rng.choice([0, 0, 1, 4, 16, 100])
    while True:
        c["lo"] = max(1, int(round(c["hi"] ** share)))
        if op == "evict":
            c["keep"] = max(1, int(c["hi"] * (0.05 + 0.9 * wide)))
            c["last"] = min(int(c["keep"] * 0.5 * far), 2000)
            c["first"] = min(c["first"], c["keep"] - c["last"])
            c["new"], c["pad"] = 1, 0
        else:
            c["new"] = {"one": 1, "some": min(some, c["lo"]), "all": 0}[kind]
            c["window"] = ALL if wide < 0.4 else max(1, int(round(c["hi"] ** far)))
        if all(x <= y for x, y in zip(_cost(c), most)):
            break
        c["batch"], c["hi"] = max(1, c["batch"] // 2), max(2, c["hi"] * 3 // 4)
    if op == "evict" or rng.random() < 0.2:
        c["bounds"] = op == "evict" and rng.random() < 0.6
    return c


def _lengths(c):
    """Rows per (sequence, head), flat: spread evenly between lo and hi, the longest first."""
    n = c["batch"] * c["hkv"]
    turn = [u if c["per_head"] else u // c["hkv"] for u in range(n)]
    return [int(round(c["hi"] - (c["hi"] - c["lo"]) * (t * 0.6180339887498949 % 1.0))) for t in turn]


def _counts(c):
    return [x if c["new"] == 0 else min(x, c["new"]) for x in _lengths(c)]


def _keeps(c):
    """Rows that a head keeps."""
    return [min(x, max(1, x * c["keep"] // c["hi"])) for x in _lengths(c)]


def _pages(c, rows):
    return [-(-x // c["page"]) for x in rows]


def _max_pages(c):
    return max(max(_pages(c, _lengths(c))), 1) + 1          # room to grow


def _row_bytes(c):
    return c["d"] * 5 // 8 if c["fmt"] == "4bit" else c["d"] * (2 if c["dtype"] == "bf16" else 4)


def _query_rows(c):
    """First row of every (sequence, head) among the queries, and their number.  Heads of unequal count start together."""
    counts, h, starts, at = _counts(c), c["hkv"], [], 0
    for b in range(c["batch"]):
        starts += [at] * h
        at += max(counts[b * h:(b + 1) * h])
    return starts, at + c["pad"]


# ------------------------------------------------------------------------------------------------- 4-bit pages
_PLACES = [(e >> 1) + 4 * (e & 1) for e in range(8)]         # nibble of element e of a run of eight


def _nibbles_out(w):
    """int32 [...] -> [..., 8] codes."""
    return (w[..., None] >> torch.tensor([4 * p for p in _PLACES], dtype=torch.int32, device=w.device)) & 15


def _values(code, step, base):
    """The elements that codes stand for, fp32."""
    s, b = step.float()[..., None], base.float()[..., None]
    return (b + s * (1.0 + code.float().unflatten(-1, (-1, 32)) / 16.0)).flatten(-2)


def _unpack_keys(pages, p, d):
    n = pages.shape[0]
    order = [0, 2, 1, 3] if d == 128 else [0, 1]             # place of each group of 32 elements in a stored key row
    w = pages[:, :p * d // 2].contiguous().view(torch.int32).view(n, p, 4, d // 32)
    code = _nibbles_out(w).transpose(2, 3)[:, :, order].reshape(n, p, d)
    sb = pages[:, p * d // 2:].contiguous().view(torch.float16).view(n, p, d // 32, 2)[:, :, order]
    return code, sb[..., 0], sb[..., 1]


def _unpack_values(pages, p, d):
    n = pages.shape[0]
    w = pages[:, :p * d // 2].contiguous().view(torch.int32).view(n, p // 32, 4, d // 64, 16, 4)
    code = _nibbles_out(w).view(n, p // 32, 4, d // 64, 16, 4, 4, 2).permute(0, 1, 7, 2, 6, 3, 5, 4).reshape(n, p, d)
    sb = pages[:, p * d // 2:].contiguous().view(torch.float16).view(n, p // 32, 4, d // 32, 2, 4, 2).permute(0, 1, 6, 2, 5, 3, 4)
    sb = sb.reshape(n, p, d // 32, 2)
    return code, sb[..., 0], sb[..., 1]


def _pool_values(c, pages, keys):
    """Every row of a pool, fp32 [pages, P, D]."""
    if c["fmt"] == "rows":
        return pages.float()
    return _values(*(_unpack_keys if keys else _unpack_values)(pages, c["page"], c["d"]))


# ------------------------------------------------------------------------------------------------- inputs
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _pool(c, g, n_pages, keys):
    """Pages as a program has filled them.  In 4 bits: bell-shaped codes, steps and bases of 32 such elements."""
    d, p = c["d"], c["page"]
    if c["fmt"] == "rows":
        x = torch.randn((n_pages, p, d), generator=g, device=DEV)
        return (x + _mean(c) if keys else x).to(_dtype(c)).contiguous()
    code = (torch.randn((n_pages, p * d), generator=g, device=DEV) * 3.6 + 7.5).round().clamp(0, 15).to(torch.uint8)
    step = 4.4 + 0.5 * torch.rand((n_pages, p * d // 32), generator=g, device=DEV)
    base = -1.46875 * step + 0.3 * torch.randn((n_pages, p * d // 32), generator=g, device=DEV)
    if keys:                                                 # (S, B) next to one another; for values eight steps, then eight bases
        sb = torch.stack((step, base), -1)
    else:
        sb = torch.stack((step.view(n_pages, -1, 8), base.view(n_pages, -1, 8)), 2)
    return torch.cat((code[:, 0::2] | code[:, 1::2] << 4, sb.half().contiguous().view(n_pages, -1).view(torch.uint8)), 1).contiguous()


def _mean(c):
    """What the keys of a head have in common."""
    x = torch.cos(torch.arange(c["d"], device=DEV) * 2.3)
    return 7.4 * x / x.norm()


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed * 2 + 1)
    rand = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    t, d, p, units, width = _dtype(c), c["d"], c["page"], c["batch"] * c["hkv"], _max_pages(c)
    lengths = _lengths(c)
    used = _pages(c, lengths)
    fresh = _pages(c, _keeps(c)) if c["op"] == "evict" else [0] * units
    n_pages = sum(used) + sum(fresh) + 3
    # pages of a head lie anywhere in the pool; what the table holds behind a head's last page is no page
    place = torch.randperm(n_pages, generator=g, device=DEV).int()

    def table_of(n, skip):
        n = i32(n)
        ordinal = skip + torch.arange(width, device=DEV)[None] + (n.cumsum(0) - n)[:, None]
        rows = torch.where(torch.arange(width, device=DEV)[None] < n[:, None], place[ordinal.clamp(max=n_pages - 1)], -1)
        return rows.int().view(c["batch"], c["hkv"], width).contiguous()

    s = dict(case=c, n_pages=n_pages, lengths=i32(lengths).view(c["batch"], -1), table=table_of(used, 0), K_pages=_pool(c, g, n_pages, True),
             scale=1.0 / math.sqrt(d))
    if c["op"] != "weights":
        s["V_pages"] = _pool(c, g, n_pages, False)
    if c["op"] == "evict":
        # what decoding leaves: a few rows with most of the weight, some with none yet
        s["weights"] = (torch.exp(2.0 * rand(n_pages, p)) * (torch.rand((n_pages, p), generator=g, device=DEV) < 0.9)).contiguous()
        s.update(into=table_of(fresh, sum(used)), into_lengths=torch.zeros_like(s["lengths"]), keep=i32(_keeps(c)).view(c["batch"], -1))
        s["kept"] = torch.empty((c["batch"], c["hkv"], max(_keeps(c))), dtype=torch.int32, device=DEV)
        if c["bounds"]:
            far = rand(n_pages, d).abs() + 0.7
            s["K_bounds"] = torch.stack((-far, far), 1).to(t).contiguous()
        if c["fmt"] == "4bit":
            rows = units * max(_keeps(c))
            s.update(K_back=torch.zeros((rows, 1, d), dtype=t, device=DEV), V_back=torch.zeros((rows, 1, d), dtype=t, device=DEV),
                     back_start=(torch.arange(units, device=DEV) * max(_keeps(c))).int().view(c["batch"], -1).contiguous())
    else:
        starts, n_rows = _query_rows(c)
        s.update(row_start=i32(starts).view(c["batch"], -1), row_count=i32(_counts(c)).view(c["batch"], -1))
        s["Q"] = (2.0 * rand(n_rows, c["hq"], d)).to(t)
        if c["op"] == "attention":
            s.update(out=torch.zeros_like(s["Q"]), lse=torch.zeros((n_rows, c["hq"]), device=DEV))
        else:
            # log-sum-exp as the attention left it: logits spread by the query's length around its product with what keys share
            at = torch.full((n_rows,), 1.0, device=DEV)
            for b in range(c["batch"]):
                n, m = _counts(c)[b * c["hkv"]], lengths[b * c["hkv"]]
                at[starts[b * c["hkv"]]:][:n] = torch.arange(m - n, m, device=DEV) + 1.0
            q = s["Q"].float()
            s["lse"] = torch.log(at.clamp(max=c["window"] + c["first"]))[:, None] + q.square().sum(-1) / (2 * d) + (q @ _mean(c) / math.sqrt(d) if c["fmt"] == "rows" else 0.0)
            s["weights"] = torch.exp(rand(n_pages, p)).contiguous()
    if own:
        s["call"] = _calls(s)                               # the argument structs that such a program builds once
    return s


def _calls(s):
    """What a serving loop holds over its buffers: the arguments of its calls, marshalled."""
    from paper_2510_20707_amd import binding as B
    c = s["case"]
    p = B.make_paged_params(c["dtype"], c["fmt"], c["batch"], c["hq"], c["hkv"], c["d"], c["page"], s["table"].shape[2], s["n_pages"], s["scale"])
    cache = B.PagedCache(s["K_pages"], s.get("V_pages"), s["table"], s["lengths"], s.get("K_bounds"))
    if c["op"] == "evict":
        into = B.PagedCache(s["K_pages"], s["V_pages"], s["into"], s["into_lengths"], s.get("K_bounds"))
        calls = (B.PreparedPagedEvict(p, [cache], [into], [s["weights"]], [s["keep"]], [s["kept"]], keep_first=c["first"], keep_last=c["last"],
                                      weights_into=[s["weights"]], max_rows=c["hi"]),)
        if c["fmt"] == "4bit":
            back = B.PagedRows(*(s[k].expand(-1, c["hkv"], -1) for k in ("K_back", "V_back")), s["back_start"], s["into_lengths"])
            calls += (B.PreparedPagedRead(p, [into], [back], max_count=max(_keeps(c))),)
        return calls
    rows = B.PagedQueries(s["Q"], s["row_start"], s["row_count"], s.get("out"), s["lse"])
    sizes = dict(window=c["window"], keep_first=c["first"], max_count=max(_counts(c)), max_rows=c["hi"])
    if c["op"] == "attention":
        return (B.PreparedPagedWindowAttention(p, [cache], [rows], **sizes),)
    return (B.PreparedPagedWeights(p, [cache], [rows], [s["weights"]], **sizes),)


# ------------------------------------------------------------------------------------------------- one pass
def run(state):
    s = state
    op = s["case"]["op"]
    if own:
        for call in s["call"]:
            call.run()
    else:
        {"attention": _attention, "weights": _weights, "evict": _evict}[op](s)
    if op == "attention":
        return {"out": s["out"], "lse": s["lse"]}
    if op == "weights":
        return {"weights": s["weights"]}
    names = ("K_back", "V_back") if s["case"]["fmt"] == "4bit" else ("K_pages", "V_pages")
    return {k: s[k] for k in names + ("weights", "K_bounds", "kept", "into_lengths") if k in s}


def _dense(s, pages, keys):
    """The rows of every (sequence, head) in order, fp32 [units, rows, D]."""
    c = s["case"]
    n = -(-c["hi"] // c["page"])
    ids = s["table"].view(-1, s["table"].shape[2])[:, :n].clamp(min=0).long()
    return _pool_values(c, pages, keys)[ids].flatten(1, 2)[:, :c["hi"]]


def _blocks(s):
    """Blocks of queries: their rows [units, block], which of them exist, the heads, the queries [units, block G, D] in fp32, and which of
    the cached rows each of them sees [units, block, rows]."""
    c = s["case"]
    units, g, most = c["batch"] * c["hkv"], c["hq"] // c["hkv"], max(_counts(c))
    count, length, start = (s[k].view(-1, 1).long() for k in ("row_count", "lengths", "row_start"))
    head = (torch.arange(units, device=DEV) % c["hkv"])[:, None]
    q = s["Q"].view(s["Q"].shape[0], c["hkv"], g, c["d"])
    j = torch.arange(c["hi"], device=DEV)
    step = max(1, min(most, BLOCK // (units * g * c["hi"])))
    for t0 in range(0, most, step):
        t = torch.arange(t0, min(most, t0 + step), device=DEV)[None]
        live = t < count
        row = torch.where(live, start + t, 0)
        place = torch.where(live, length - count + t, -1)[:, :, None]
        sees = (j <= place) & ((j > place - c["window"]) | (j < c["first"]))
        yield row, live, head.expand_as(row), q[row, head].float().flatten(1, 2), sees


def _attention(s):
    c = s["case"]
    g, d = c["hq"] // c["hkv"], c["d"]
    k, v = _dense(s, s["K_pages"], True).transpose(1, 2).contiguous(), _dense(s, s["V_pages"], False)
    out, lse = s["out"].view(-1, c["hkv"], g, d), s["lse"].view(-1, c["hkv"], g)
    for row, live, head, q, sees in _blocks(s):
        x = (torch.bmm(q, k) * s["scale"]).unflatten(1, (-1, g))
        x.masked_fill_(~sees[:, :, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        w = x.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
        total = w.sum(-1, keepdim=True)
        o = torch.bmm(w.flatten(1, 2), v).view(*w.shape[:3], d) / torch.where(total > 0, total, 1.0)
        out[row[live], head[live]] = o[live].to(out.dtype)
        lse[row[live], head[live]] = (top + total.log())[..., 0][live]


def _weights(s):
    c = s["case"]
    g, p = c["hq"] // c["hkv"], c["page"]
    k = _dense(s, s["K_pages"], True).transpose(1, 2).contiguous()
    units, rows = k.shape[0], k.shape[2]
    lse, got = s["lse"].view(-1, c["hkv"], g), torch.zeros((units, rows), dtype=torch.float64, device=DEV)
    for row, live, head, q, sees in _blocks(s):
        x = (torch.bmm(q, k) * s["scale"]).unflatten(1, (-1, g)).sub_(lse[row, head][..., None]).exp_()
        got += x.masked_fill_(~sees[:, :, None], 0.0).sum((1, 2), dtype=torch.float64)
    j = torch.arange(rows, device=DEV)[None].expand(units, -1)
    length, count = s["lengths"].view(-1, 1).long(), s["row_count"].view(-1, 1).long()
    there = j < length
    page = s["table"].view(units, -1).gather(1, j // p)[there].long()
    old = s["weights"][page, (j % p)[there]].double()
    s["weights"][page, (j % p)[there]] = (torch.where((j >= length - count)[there], 0.0, old) + got[there]).float()


def _ranked(s, weight):
    """Which rows [units, rows] are kept, by the weights of all."""
    c = s["case"]
    j = torch.arange(weight.shape[1], device=DEV)[None]
    length, keep = s["lengths"].view(-1, 1), s["keep"].view(-1, 1)
    x = torch.where((j < c["first"]) | (j >= length - c["last"]), math.inf, weight)
    x = torch.where(j < length, x, -math.inf)
    order = x.sort(dim=1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(1, order, j.expand_as(order))
    return (rank < keep) & (j < length)


def _evict(s):
    c = s["case"]
    p, units = c["page"], c["batch"] * c["hkv"]
    n = -(-c["hi"] // p)
    table, into = s["table"].view(units, -1), s["into"].view(units, -1)
    kept = _ranked(s, s["weights"][table[:, :n].clamp(min=0).long()].flatten(1)[:, :c["hi"]])
    u, j = kept.nonzero(as_tuple=True)
    count = kept.sum(1)
    i = torch.arange(u.numel(), device=DEV) - (count.cumsum(0) - count)[u]            # place in what is left
    at, to = (table[u, j // p].long(), j % p), (into[u, i // p].long(), i % p)
    s["into_lengths"].copy_(count.view_as(s["into_lengths"]))
    s["kept"].fill_(-1).view(units, -1)[u, i] = j.int()
    s["weights"][to] = s["weights"][at]
    if c["fmt"] == "rows":
        s["K_pages"][to] = s["K_pages"][at]
        s["V_pages"][to] = s["V_pages"][at]
        k = s["K_pages"][to].float()
    else:
        k = _pool_values(c, s["K_pages"], True)[at].to(_dtype(c))
        row = u * s["kept"].shape[2] + i
        s["K_back"][row, 0] = k
        s["V_back"][row, 0] = _pool_values(c, s["V_pages"], False)[at].to(_dtype(c))
        k = k.float()
    if c["bounds"]:
        both = s["K_bounds"].float()
        both[to[0]] = torch.tensor([math.inf, -math.inf], device=DEV)[:, None].expand(2, c["d"])
        idx = to[0][:, None].expand(-1, c["d"])
        both[:, 0].scatter_reduce_(0, idx, k, "amin")
        both[:, 1].scatter_reduce_(0, idx, k, "amax")
        s["K_bounds"].copy_(both)


# ------------------------------------------------------------------------------------------------- what it cannot do without
def _seen(c, length, count):
    """Pairs of a new row and a cached row that it sees, and cached rows that any of them sees."""
    w, f = c["window"], c["first"]
    lo = length - count

    def up_to(n, w):                                         # sum of min(place + 1, w) over the places below n
        k = min(n, w)
        return k * (k + 1) // 2 + (n - k) * w

    pairs = up_to(length, w) - up_to(lo, w)
    pairs += sum(min(f, max(0, x - w + 1)) for x in range(max(lo, w), min(length, w + f))) + f * max(0, length - max(lo, w + f)) if f else 0
    return pairs, min(length, max(0, length - max(0, lo - w + 1)) + min(f, max(0, lo - w + 1)))


def work(case):
    c = case
    e, d, h, units = (2 if c["dtype"] == "bf16" else 4), c["d"], c["hkv"], c["batch"] * c["hkv"]
    if c["op"] == "evict":
        keeps = _keeps(c)
        moved, rows = sum(keeps), sum(_lengths(c))
        n = {"bytes": 4 * rows + 4 * sum(_pages(c, _lengths(c))) + moved * (4 * _row_bytes(c) + 8) + 4 * units * max(keeps), "flops": rows}
        if c["bounds"]:
            n["bytes"] += sum(_pages(c, keeps)) * 2 * d * e
        if c["fmt"] == "4bit":
            n["bytes"] += 2 * moved * (_row_bytes(c) + d * e)
        return n
    pairs, rows = (sum(x) for x in zip(*(_seen(c, n, m) for n, m in zip(_lengths(c), _counts(c)))))
    queries = sum(_counts(c)) * (c["hq"] // h)
    if c["op"] == "weights":
        return {"bytes": rows * (_row_bytes(c) + 8) + queries * (d * e + 4), "flops": 2 * pairs * d * (c["hq"] // h)}
    return {"bytes": 2 * rows * _row_bytes(c) + queries * (2 * d * e + 4), "flops": 4 * pairs * d * (c["hq"] // h)}


# ------------------------------------------------------------------------------------------------- 64 bits, from the definitions
def _stored(c, pages, keys):
    """Every element of a pool by its own address: which byte holds its code, which two fp16 its group's step and base."""
    if c["fmt"] == "rows":
        return pages.double()
    p, d = c["page"], c["d"]
    r, e = torch.arange(p, device=DEV)[:, None], torch.arange(d, device=DEV)[None]
    grp, n = e // 32, d // 32
    if keys:
        place = (grp % 2) * 2 + grp // 2 if d == 128 else grp
        word = r * (d // 8) + (e % 32 // 8) * n + place
        i = e % 8
        scale = (r * n + place) * 2
        gap = 1
    else:
        strip = r // 32 * 4 + r % 16 // 4
        word = strip * d + e // 64 * 64 + e % 16 * 4 + e // 16 % 4
        i = r % 4 * 2 + r % 32 // 16
        scale = (strip * n + grp) * 16 + i
        gap = 8
    nib = i // 2 + 4 * (i % 2)
    byte = pages[:, (word * 4 + nib // 2).flatten()].view(-1, p, d).int()
    code = (byte >> (4 * (nib % 2)).int()) % 16
    half = pages[:, p * d // 2:].contiguous().view(torch.float16).double()
    step, base = half[:, scale.expand(p, d).flatten()].view(-1, p, d), half[:, (scale + gap).expand(p, d).flatten()].view(-1, p, d)
    return base + step * (1.0 + code.double() / 16.0)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    units, d, p, h = c["batch"] * c["hkv"], c["d"], c["page"], c["hkv"]
    g, table, lengths = c["hq"] // h, s["table"].view(units, -1).long(), _lengths(c)
    kk = _stored(c, s["K_pages"], True)
    vv = _stored(c, s["V_pages"], False) if c["op"] != "weights" else None
    if c["op"] == "evict":
        got = {k: s[k].double() for k in ("K_pages", "V_pages", "K_back", "V_back", "weights", "K_bounds") if k in s and s[k].dtype != torch.uint8}
        into, keeps = s["into"].view(units, -1).long(), _keeps(c)
        for u in range(units):
            j = torch.arange(lengths[u], device=DEV)
            w = s["weights"][table[u, j // p], j % p].double()
            w[:c["first"]] = math.inf
            w[max(0, lengths[u] - c["last"]):] = math.inf
            j = (-w).sort(stable=True).indices[:keeps[u]].sort().values
            i = torch.arange(j.numel(), device=DEV)
            at, to = (table[u, j // p], j % p), (into[u, i // p], i % p)
            got["weights"][to] = s["weights"][at].double()
            if c["fmt"] == "rows":
                got["K_pages"][to], got["V_pages"][to] = kk[at], vv[at]
            else:
                rows = u * s["kept"].shape[2] + i
                got["K_back"][rows, 0], got["V_back"][rows, 0] = kk[at], vv[at]
            if c["bounds"]:
                n = -(-j.numel() // p) * p
                k = torch.cat((kk[at], kk[at][-1:].expand(n - j.numel(), -1))).view(-1, p, d)   # a page's rows, the last one repeated
                ids = into[u, :n // p]
                got["K_bounds"][ids, 0], got["K_bounds"][ids, 1] = k.amin(1), k.amax(1)
        return got
    out = torch.zeros((s["Q"].shape[0], c["hq"], d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["Q"].shape[0], c["hq"]), dtype=torch.float64, device=DEV)
    if c["op"] == "weights":
        lse, weights = s["lse"].double(), s["weights"].double()
    starts, _ = _query_rows(c)
    for u in range(units):
        n, m, heads = lengths[u], _counts(c)[u], slice(u % h * g, (u % h + 1) * g)
        j = torch.arange(n, device=DEV)
        k = kk[table[u, j // p], j % p].t().contiguous()
        v = vv[table[u, j // p], j % p] if vv is not None else None
        got = torch.zeros(n, dtype=torch.float64, device=DEV)
        step = max(1, 2 ** 28 // (g * n))
        for t in range(0, m, step):
            rows = slice(starts[u] + t, starts[u] + min(m, t + step))
            q = s["Q"][rows, heads].double()                                      # [block, G, D]
            place = n - m + torch.arange(t, min(m, t + step), device=DEV)
            hidden = (j[None] > place[:, None]) | ((j[None] <= place[:, None] - c["window"]) & (j[None] >= c["first"]))
            x = (q @ k * s["scale"]).masked_fill(hidden[:, None], -math.inf)
            if c["op"] == "weights":
                got += torch.exp(x - lse[rows, heads][..., None]).sum((0, 1))
            else:
                lse[rows, heads] = torch.logsumexp(x, -1)
                out[rows, heads] = torch.softmax(x, -1) @ v
        if c["op"] == "weights":
            at = (table[u, j // p], j % p)
            weights[at] = torch.where(j < n - m, weights[at], 0.0) + got
    return {"weights": weights} if c["op"] == "weights" else {"out": out, "lse": lse}

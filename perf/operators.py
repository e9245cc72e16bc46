"""The operators on a paged cache, measured: what a serving program does with a compacted or full cache that goes on
growing, page by page, after the prefill.

  append     new key and value rows rotated to their positions (queries too, in the same pass) and written into the pages
             of every head, in the rows' own type or in 4 bits, with the pages' key bounds
  read       rows of the pages back in dense form (a cache that is compressed again, or moved)
  select     for every new token and KV head the pages with the largest upper bound of the attention scores
  attention  of one new token per sequence over its pages, all of them or the selected ones

A page holds `page` rows of one KV head; a head's pages come from a table [batch, hkv, pages]; heads of one sequence may
have different lengths (head-adaptive budgets).  4-bit rows: 32 neighbouring elements share a step S and a base B, both
fp16, and an element is B + S (1 + code / 16).

A case is a dict of plain values.  `own` False: elementary torch operations; True: the library's entry points.
"""
import math

import torch

own = False

DEV = "cuda:0"
CLIP = 16384.0               # elements beyond it are stored as it in 4 bits
THETA = 1.0e6


# ------------------------------------------------------------------------------------------------- the cases
def _case(op, **kw):
    """lo, hi: rows of the shortest and the longest sequence (or head, with per_head), those being appended among them;
    new: rows appended or read per head, 0: all of them; axes: 0 no rotation, 1 one position per token, 3 one for time, height and
    width each; pad: rows behind the last sequence; keep: pages selected."""
    c = dict(op=op, fmt="4bit", dtype="bf16", batch=1, hq=28, hkv=4, d=128, page=64, lo=8192, hi=8192, per_head=False, new=1,
             axes=1, bounds=False, fused=True, pad=0, keep=0)
    c.update(kw)
    return c


def listed():
    return [
        # one decoding step's rows of one sequence, rotated by the three axes of a vision-language model, full precision: latency
        _case("append", name="append_step_one", fmt="rows", axes=3, lo=8193, hi=8193),
        # the same for a batch of 64 sequences of unequal length into 4-bit pages, and what was stored read back
        _case("append", name="append_step_batch_4bit", batch=64, hq=32, hkv=8, lo=1, hi=16384, bounds=True),
        # four prompts of 5 to 32 thousand tokens straight into 4-bit pages, in a batch padded at its end, and read back
        _case("append", name="append_prompts_4bit", batch=4, lo=5001, hi=32768, new=0, axes=3, bounds=True, pad=77),
        # a compacted fp32 cache of a small model moved into pages, heads of unequal length, no rotation
        _case("append", name="append_compacted_f32", fmt="rows", dtype="f32", batch=2, hq=16, hkv=8, d=64, page=32, lo=33, hi=700,
              per_head=True, new=0, axes=0, fused=False, bounds=True),
        # the newest 64 rows of eight sequences, full precision
        _case("read", name="read_window_rows", fmt="rows", batch=8, hq=32, hkv=8, lo=64, hi=4000, new=64),
        # a whole 4-bit cache of four long sequences in dense form, to be compressed again
        _case("read", name="read_cache_4bit", batch=4, lo=8192, hi=32768, new=0),
        # pages for one sequence of 131072 tokens
        _case("select", name="select_one_131k", lo=131072, hi=131072, keep=64, bounds=True),
        # pages of 32 rows for a batch of 32 sequences
        _case("select", name="select_batch", batch=32, hq=32, hkv=8, page=32, lo=3000, hi=32768, keep=128, bounds=True),
        # one sequence right after compression to 128 rows a head on average: latency
        _case("attention", name="attention_one_4bit", lo=48, hi=260, per_head=True, page=32),
        # a decoding step of 64 sequences of 1 to 16384 tokens on 4-bit pages
        _case("attention", name="attention_batch_4bit", batch=64, hq=32, hkv=8, lo=1, hi=16384),
        # 16 sequences of 32 thousand tokens, 64 selected pages of each
        _case("attention", name="attention_sparse_4bit", batch=16, lo=30000, hi=32768, keep=64),
        # full-precision pages, eight sequences
        _case("attention", name="attention_rows", fmt="rows", batch=8, hq=16, hkv=8, d=64, lo=1000, hi=16384),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case of the same ranges: one to 64 sequences of one to 131072 rows, both formats and types, pages of 32 to 128."""
    op = rng.choice(["append", "append", "read", "select", "attention", "attention", "attention"])
    hq, hkv = rng.choice([(28, 4), (32, 8), (16, 8), (12, 2), (4, 2), (40, 8), (8, 8), (32, 2)])
    d = rng.choice([128, 128, 64])
    fmt, dtype = rng.choice([("4bit", "bf16")] * 3 + [("rows", "bf16"), ("rows", "f32")])
    batch = _log(rng, 1, 64)
    hi = _log(rng, 1024 if op == "select" else 1, 131072)
    # no dearer than the largest listed case of the operator
    most = {"append": 4 * 4 * 20000, "read": 4 * 4 * 20000, "select": 32 * 8 * 18000, "attention": 64 * 8 * 8000}[op]
    if fmt == "rows":
        most //= 8 if dtype == "f32" else 4
    every = op == "append" and rng.random() < 0.5 or op == "read" and rng.random() < 0.7
    if op == "append" and not every:
        most = 64 * 8 * 8000 // (8 if dtype == "f32" else 2)
    while batch * hkv * hi > most:
        batch, hi = max(1, batch // 2), hi * 3 // 4
    lo = _log(rng, 1, hi)
    page = rng.choice([32, 64, 64, 128])
    new = 0 if every else min(lo, _log(rng, 1, 100))
    fused = op == "append" and rng.random() < 0.7
    pages = -(-hi // page)
    keep = 0
    if op == "select":
        keep = _log(rng, 3, min(256, pages - 1))             # more pages than that: something to choose
    elif op == "attention" and rng.random() < 0.4:
        keep = _log(rng, 1, min(256, pages))
    return _case(op, fmt=fmt, dtype=dtype, batch=batch, hq=hq, hkv=hkv, d=d, page=page, lo=lo, hi=hi,
                 per_head=rng.random() < 0.4 and not (fused and op == "append"), new=new,
                 axes=rng.choice([0, 1, 3]) if fused else 0, bounds=op == "select" or op == "append" and rng.random() < 0.5,
                 fused=fused, pad=rng.choice([0, 0, 5, 64]) if fused else 0, keep=keep)


def _lengths(c):
    """Rows per (sequence, head), flat: spread evenly between lo and hi, the longest first."""
    n = c["batch"] * c["hkv"]
    turn = [u if c["per_head"] else u // c["hkv"] for u in range(n)]
    return [int(round(c["hi"] - (c["hi"] - c["lo"]) * (t * 0.6180339887498949 % 1.0))) for t in turn]


def _counts(c):
    return [x if c["new"] == 0 else min(x, c["new"]) for x in _lengths(c)]


def _pages_of(c):
    return [-(-x // c["page"]) for x in _lengths(c)]


def _max_pages(c):
    return max(max(_pages_of(c)), 1) + 1                    # room to grow


def _row_bytes(c):
    if c["fmt"] == "4bit":
        return c["d"] * 5 // 8                              # codes, and two fp16 for 32 elements
    return c["d"] * (2 if c["dtype"] == "bf16" else 4)


def _source_rows(c):
    """First row of every (sequence, head) in the dense tensor, and that tensor's rows: tokens one after another, or
    (not fused) each head's rows in a block of their own."""
    counts, h = _counts(c), c["hkv"]
    if c["fused"]:
        starts, at = [], 0
        for b in range(c["batch"]):
            starts += [at] * h
            at += counts[b * h]
        return starts, at + c["pad"]
    block = max(counts)
    return [u * block for u in range(len(counts))], len(counts) * block + c["pad"]


def _chosen(c):
    """Pages an attention over `keep` selected pages reads, per (sequence, head)."""
    return [min(n, c["keep"]) if c["keep"] else n for n in _pages_of(c)]


# ------------------------------------------------------------------------------------------------- 4-bit rows
def _quantise(x):
    """Codes (int32), steps and bases (fp16) of the rows of x [..., D], decided in 64 bits."""
    g = x.double().clamp(-CLIP, CLIP).unflatten(-1, (-1, 32))
    lo, hi = g.amin(-1), g.amax(-1)
    step = ((hi - lo) * (16.0 / 15.0)).float().half()
    base = (lo - step.double()).float().half()
    s, b = step.double()[..., None], base.double()[..., None]
    code = torch.where(s > 0, ((g - b - s) * 16.0 / torch.where(s > 0, s, 1.0)).round().clamp(0, 15), 0.0)
    return code.int().flatten(-2), step, base


def _values(code, step, base):
    """The elements that codes stand for, fp32."""
    s, b = step.float()[..., None], base.float()[..., None]
    return (b + s * (1.0 + code.float().unflatten(-1, (-1, 32)) / 16.0)).flatten(-2)


_PLACES = [(e >> 1) + 4 * (e & 1) for e in range(8)]         # nibble of element e of a run of eight


def _nibbles_in(x):
    """[..., 8] codes -> int32 [...]."""
    v = (x.long() << torch.tensor([4 * p for p in _PLACES], device=x.device)).sum(-1)
    return torch.where(v >= 2 ** 31, v - 2 ** 32, v).int()


def _nibbles_out(w):
    """int32 [...] -> [..., 8] codes."""
    return (w[..., None] >> torch.tensor([4 * p for p in _PLACES], dtype=torch.int32, device=w.device)) & 15


def _order(d):
    """Place of each group of 32 elements in a stored key row."""
    half = max(1, d // 64)
    return [(c % half) * 2 + c // half for c in range(d // 32)] if d == 128 else list(range(d // 32))


def _pack_keys(code, step, base):
    """[pages, P, D] codes -> uint8 pages.  A row's word (run, place): the eight elements 32 group + 8 run + e."""
    n, p, d = code.shape
    back = sorted(range(d // 32), key=_order(d).__getitem__)
    w = _nibbles_in(code.view(n, p, d // 32, 4, 8)[:, :, back].transpose(2, 3).contiguous())
    sb = torch.stack((step, base), -1)[:, :, back].contiguous()
    return torch.cat((w.view(n, -1).view(torch.uint8), sb.view(n, -1).view(torch.uint8)), 1)


def _unpack_keys(pages, p, d):
    n = pages.shape[0]
    order = _order(d)
    w = pages[:, :p * d // 2].contiguous().view(torch.int32).view(n, p, 4, d // 32)
    code = _nibbles_out(w).transpose(2, 3)[:, :, order].reshape(n, p, d)
    sb = pages[:, p * d // 2:].contiguous().view(torch.float16).view(n, p, d // 32, 2)[:, :, order]
    return code, sb[..., 0], sb[..., 1]


def _pack_values(code, step, base):
    """Tiles of 32 rows in four strips: strip q holds the rows 4 q .. 4 q + 3 and 16 + 4 q .. 16 + 4 q + 3, one word of eight codes per
    element, the elements in the order 64 j + 16 w + i at word 64 j + 4 i + w."""
    n, p, d = code.shape
    w = _nibbles_in(code.view(n, p // 32, 2, 4, 4, d // 64, 4, 16).permute(0, 1, 3, 5, 7, 6, 4, 2).reshape(n, p // 32, 4, d, 8))
    sb = torch.stack((step, base), -1).view(n, p // 32, 2, 4, 4, d // 32, 2).permute(0, 1, 3, 5, 6, 4, 2).contiguous()
    return torch.cat((w.view(n, -1).view(torch.uint8), sb.view(n, -1).view(torch.uint8)), 1)


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


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed * 2 + 1)
    rand = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    t, d, p, units = _dtype(c), c["d"], c["page"], c["batch"] * c["hkv"]
    used, width = _pages_of(c), _max_pages(c)
    n_pages = sum(used) + 3
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    lengths, counts = i32(_lengths(c)).view(c["batch"], -1), i32(_counts(c)).view(c["batch"], -1)
    # pages of a head lie anywhere in the pool; what the table holds behind a head's last page is no page
    place = torch.randperm(n_pages, generator=g, device=DEV).int()
    n_used = i32(used)
    ordinal = torch.arange(width, device=DEV)[None] + (n_used.cumsum(0) - n_used)[:, None]
    table = torch.where(torch.arange(width, device=DEV)[None] < n_used[:, None], place[ordinal.clamp(max=n_pages - 1)], -1).int()
    s = dict(case=c, lengths=lengths, table=table.view(c["batch"], c["hkv"], width).contiguous(), n_pages=n_pages)
    mean = rand(d)
    mean = mean / mean.norm()
    if c["op"] != "select":
        k, v = (rand(n_pages, p, d) + 7.4 * mean).to(t), rand(n_pages, p, d).to(t)
        if c["fmt"] == "4bit":
            k, v = _pack_keys(*_quantise(k)), _pack_values(*_quantise(v))
        s.update(K_pages=k.contiguous(), V_pages=v.contiguous())
    if c["bounds"]:
        mid, far = rand(n_pages, d) * 0.5 + 7.4 * mean, rand(n_pages, d).abs() + 0.7
        s["K_bounds"] = torch.stack((mid - far, mid + far), 1).to(t).contiguous()
    if c["op"] in ("append", "read"):
        starts, n_rows = _source_rows(c)
        s.update(row_start=i32(starts).view_as(lengths), row_count=counts)
        blank = lambda *shape: torch.zeros(shape, dtype=t, device=DEV)  # noqa: E731
        if c["op"] == "append" and c["fused"]:
            x = rand(n_rows, c["hq"] + 2 * c["hkv"], d).to(t)          # one projection's output: queries, keys, values
            s.update(Q=x[:, :c["hq"]], K=x[:, c["hq"]:c["hq"] + c["hkv"]], V=x[:, c["hq"] + c["hkv"]:], Q_out=blank(n_rows, c["hq"], d))
        elif c["op"] == "append":
            s.update(K=(rand(n_rows, 1, d) + 7.4 * mean).to(t).expand(-1, c["hkv"], -1), V=rand(n_rows, 1, d).to(t).expand(-1, c["hkv"], -1))
        if c["op"] == "read" or c["fmt"] == "4bit":
            shape = (n_rows, c["hkv"], d) if c["fused"] else (n_rows, 1, d)
            s.update(K_back=blank(*shape), V_back=blank(*shape))
    if c["axes"] and c["op"] == "append":
        far = c["hi"] + 16
        angle = torch.arange(far, device=DEV, dtype=torch.float64)[:, None] * THETA ** (-torch.arange(d // 2, device=DEV, dtype=torch.float64) * 2 / d)
        s.update(cos=angle.cos().float(), sin=angle.sin().float())
        s["positions"] = torch.randint(0, far, (c["axes"], s["K"].shape[0]), generator=g, device=DEV).int()
        s["sections"] = (d // 8, 3 * d // 16, 3 * d // 16) if c["axes"] == 3 else None
    if c["op"] in ("select", "attention"):
        s["Q"] = (rand(c["batch"], c["hq"], d) * (2.0 / math.sqrt(d))).to(t)
    if c["op"] == "attention":
        s["out"] = torch.empty_like(s["Q"])
        if c["keep"]:                                                    # any ascending pages, the newest among them
            order = torch.rand(units, width, generator=g, device=DEV)
            at = torch.arange(width, device=DEV)[None]
            order = torch.where(at == n_used[:, None] - 1, 2.0, torch.where(at < n_used[:, None], order, -1.0))
            n = i32(_chosen(c))
            best = order.topk(min(c["keep"], width), 1).indices
            best = torch.where(torch.arange(best.shape[1], device=DEV)[None] < n[:, None], best, 2 ** 30).sort(1).values
            sel = torch.full((units, c["keep"]), -1, dtype=torch.int32, device=DEV)
            sel[:, :best.shape[1]] = torch.where(best < 2 ** 30, best, -1).int()
            s.update(selected=sel.view(c["batch"], c["hkv"], -1), n_selected=n.view(c["batch"], -1))
    elif c["op"] == "select":
        s["selected"] = torch.empty((c["batch"], c["hkv"], c["keep"]), dtype=torch.int32, device=DEV)
        s["n_selected"] = torch.empty((c["batch"], c["hkv"]), dtype=torch.int32, device=DEV)
    if own:
        s["call"] = _calls(s)                               # the argument structs that such a program builds once
    return s


def _calls(s):
    """What a serving loop holds over its buffers: the arguments of its calls, marshalled."""
    from paper_2510_20707_amd import binding as B
    c = s["case"]
    p = B.make_paged_params(c["dtype"], c["fmt"], c["batch"], c["hq"], c["hkv"], c["d"], c["page"], s["table"].shape[2], s["n_pages"])
    cache = B.PagedCache(s.get("K_pages"), s.get("V_pages"), s["table"], s["lengths"], s.get("K_bounds"))
    if c["op"] == "select":
        return (B.PreparedPagedSelect(p, [cache], [s["Q"]], [s["selected"]], [s["n_selected"]], keep_first=1, keep_last=1),)
    if c["op"] == "attention":
        return (B.PreparedPagedAttention(p, [cache], [s["Q"]], [s["out"]], [s["selected"]] if c["keep"] else None,
                                         [s["n_selected"]] if c["keep"] else None),)
    calls, most = (), max(_counts(c))
    if c["op"] == "append":
        rope = B.Rope(s["cos"], s["sin"], s["positions"], s["sections"]) if c["axes"] else None
        rows = B.PagedRows(s["K"], s["V"], s["row_start"], s["row_count"], s.get("Q"), s.get("Q_out"))
        calls += (B.PreparedPagedAppend(p, [cache], [rows], rope, max_count=most),)
    if c["op"] == "read" or c["fmt"] == "4bit":
        back = B.PagedRows(*(s[k].expand(-1, c["hkv"], -1) for k in ("K_back", "V_back")), s["row_start"], s["row_count"])
        calls += (B.PreparedPagedRead(p, [cache], [back], max_count=most),)
    return calls


# ------------------------------------------------------------------------------------------------- one pass
def run(state):
    s = state
    op = s["case"]["op"]
    if own:
        for call in s["call"]:
            call.run()
    else:
        {"append": _append, "read": _read, "select": _select, "attention": _attention}[op](s)
    return _results(s)


def _results(s):
    op = s["case"]["op"]
    if op == "select":
        return {"selected": s["selected"], "n_selected": s["n_selected"]}
    if op == "attention":
        return {"out": s["out"]}
    if op == "read" or s["case"]["fmt"] == "4bit":
        names = ("K_back", "V_back")
    else:
        names = ("K_pages", "V_pages")
    return {k: s[k] for k in names + (("K_bounds", "Q_out") if op == "append" else ()) if k in s}


def _rows_of(s):
    """For every appended or read row: its (sequence, head), its place in the head, its row in the dense tensor."""
    c = s["case"]
    total = sum(_counts(c))
    count = s["row_count"].view(-1).long()
    u = torch.repeat_interleave(torch.arange(count.numel(), device=DEV), count, output_size=total)
    t = torch.arange(total, device=DEV) - (count.cumsum(0) - count)[u]
    return u, s["lengths"].view(-1).long()[u] - count[u] + t, s["row_start"].view(-1).long()[u] + t


def _angles(s, rows, of):
    """cos and sin of the given rows' positions, in `of`'s type."""
    half = s["cos"].shape[1]
    if s["sections"] is None:
        axis = torch.zeros(half, dtype=torch.long, device=DEV)
    else:
        axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(s["sections"], device=DEV), output_size=half)
    at = s["positions"].long()[:, rows][axis].t()                        # [rows, D / 2]
    i = torch.arange(half, device=DEV)
    return s["cos"][at, i].to(of), s["sin"][at, i].to(of)


def _rotated(s, x, rows):
    """x [rows, heads, D], rotated in 64 bits and rounded once."""
    if "cos" not in s:
        return x
    cos, sin = (a[:, None] for a in _angles(s, rows, torch.float64))
    a, b = x.double().chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(x.dtype)


def _append(s):
    c = s["case"]
    p, t = c["page"], _dtype(c)
    u, at, row = _rows_of(s)
    h = u % c["hkv"]
    k, v = _rotated(s, s["K"][row, h][:, None], row)[:, 0], s["V"][row, h]
    page = s["table"].view(-1, s["table"].shape[2])[u, at // p].long()
    if c["fmt"] == "rows":
        s["K_pages"][page, at % p] = k
        s["V_pages"][page, at % p] = v
    else:
        hh = h if c["fused"] else torch.zeros_like(h)
        s["K_back"][row, hh] = _values(*_quantise(k)).to(t)
        s["V_back"][row, hh] = _values(*_quantise(v)).to(t)
    if "K_bounds" in s:
        fresh = page[at % p == 0]                                        # pages that begin here forget what they bounded
        limit = torch.tensor([math.inf, -math.inf], device=DEV)
        both = s["K_bounds"].float()
        both[fresh] = limit[:, None].expand(2, c["d"])
        idx = page[:, None].expand(-1, c["d"])
        both[:, 0].scatter_reduce_(0, idx, k.float(), "amin")
        both[:, 1].scatter_reduce_(0, idx, k.float(), "amax")
        s["K_bounds"].copy_(both)
    if "Q" in s:
        n = s["Q"].shape[0] - c["pad"]
        s["Q_out"][:n] = _rotated(s, s["Q"][:n], torch.arange(n, device=DEV))


def _read(s):
    c = s["case"]
    u, at, row = _rows_of(s)
    h = u % c["hkv"] if c["fused"] else torch.zeros_like(u)
    page = s["table"].view(-1, s["table"].shape[2])[u, at // c["page"]].long()
    s["K_back"][row, h] = _pool_values(c, s["K_pages"], True)[page, at % c["page"]].to(_dtype(c))
    s["V_back"][row, h] = _pool_values(c, s["V_pages"], False)[page, at % c["page"]].to(_dtype(c))


def _select(s):
    c = s["case"]
    units, width, keep = c["batch"] * c["hkv"], s["table"].shape[2], c["keep"]
    q = s["Q"].double().view(units, -1, c["d"])
    both = s["K_bounds"].double()[s["table"].view(units, width).clamp(min=0).long()]      # [units, width, 2, D]
    score = (both[:, :, 1] * q.clamp(min=0).sum(1)[:, None]).sum(-1) + (both[:, :, 0] * q.clamp(max=0).sum(1)[:, None]).sum(-1)
    score = score.float().double()                                       # ranked as 32-bit numbers, equal ones by place
    n = (s["lengths"].view(units, 1) + c["page"] - 1) // c["page"]
    at = torch.arange(width, device=DEV)[None]
    score = torch.where((at < 1) | (at >= n - 1), math.inf, score)       # the first page and the newest are always kept
    score = torch.where(at < n, score, -math.inf)
    order = score.sort(dim=1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(1, order, at.expand(units, width))
    kept = (at < n) & (rank < keep)
    place = torch.where(kept, at, 2 ** 30).sort(1).values
    place = torch.nn.functional.pad(place, (0, max(0, keep - width)), value=2 ** 30)[:, :keep]
    s["selected"].copy_(torch.where(place < 2 ** 30, place, -1).view_as(s["selected"]))
    s["n_selected"].copy_(kept.sum(1).view_as(s["n_selected"]))


def _attention(s):
    c = s["case"]
    units, width, p = c["batch"] * c["hkv"], s["table"].shape[2], c["page"]
    table, lengths = s["table"].view(units, width), s["lengths"].view(units)
    if c["keep"]:
        nth = s["selected"].view(units, -1)
        ids = torch.where(nth >= 0, table.gather(1, nth.clamp(min=0).long()), -1)
    else:
        nth, ids = torch.arange(width, device=DEV)[None].expand(units, -1), table
    row = nth[:, :, None] * p + torch.arange(p, device=DEV)
    live = ((ids >= 0)[:, :, None] & (row < lengths[:, None, None])).flatten(1)           # [units, rows]
    ids = ids.clamp(min=0).long()
    k = _pool_values(c, s["K_pages"], True)[ids].flatten(1, 2)
    v = _pool_values(c, s["V_pages"], False)[ids].flatten(1, 2)
    v = torch.where(live[..., None], v, 0.0)
    q = s["Q"].float().view(units, -1, c["d"])
    x = torch.where(live[:, None], q @ k.transpose(1, 2).contiguous(), -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    total = w.sum(-1, keepdim=True)
    out = torch.where(total > 0, (w @ v) / torch.where(total > 0, total, 1.0), 0.0)
    s["out"].copy_(out.view_as(s["out"]))


# ------------------------------------------------------------------------------------------------- what it cannot do without
def work(case):
    c = case
    e, d, h = (2 if c["dtype"] == "bf16" else 4), c["d"], c["hkv"]
    rows, counts = sum(_lengths(c)), sum(_counts(c))
    table = sum(_pages_of(c)) * 4 + 4 * c["batch"] * h
    if c["op"] == "select":
        pages = sum(_pages_of(c))
        return {"bytes": pages * 2 * d * e + table + c["batch"] * (c["hq"] * d * e + h * c["keep"] * 4), "flops": pages * 4 * d}
    if c["op"] == "attention":
        if c["keep"]:
            rows = sum(min(n * c["page"], x) for n, x in zip(_chosen(c), _lengths(c)))
            table = sum(_chosen(c)) * 8
        return {"bytes": 2 * rows * _row_bytes(c) + table + 2 * c["batch"] * c["hq"] * d * e, "flops": 4 * rows * d * (c["hq"] // h)}
    back = 2 * counts * (_row_bytes(c) + d * e)              # pages read, dense rows written
    if c["op"] == "read":
        return {"bytes": back, "flops": 2 * counts * d}
    tokens = counts // h if c["fused"] else 0
    moved = 2 * counts * (_row_bytes(c) + d * e) + 2 * tokens * c["hq"] * d * e
    if c["axes"]:
        moved += tokens * (4 * d + 4 * c["axes"])
    if c["bounds"]:
        moved += sum(-(-x // c["page"]) for x in _counts(c)) * 2 * d * e
    return {"bytes": moved + (back if c["fmt"] == "4bit" else 0), "flops": 3 * d * (counts + tokens * c["hq"])}


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
    if c["op"] == "select":
        return None                                          # whole numbers only
    s = prepare(c, seed)
    units, d, p = c["batch"] * c["hkv"], c["d"], c["page"]
    if c["op"] == "attention":
        kk, vv = _stored(c, s["K_pages"], True), _stored(c, s["V_pages"], False)
        out = torch.zeros(units, c["hq"] // c["hkv"], d, dtype=torch.float64, device=DEV)
        q = s["Q"].double().view(units, -1, d)
        n_rows, table = _lengths(c), s["table"].view(units, -1).long()
        sel = s["selected"].view(units, -1) if c["keep"] else None
        for u in range(units):
            pages = torch.arange(-(-n_rows[u] // p), device=DEV) if sel is None else sel[u][sel[u] >= 0].long()
            at = (pages[:, None] * p + torch.arange(p, device=DEV)).flatten() < n_rows[u]
            k, v = kk[table[u, pages]].reshape(-1, d)[at], vv[table[u, pages]].reshape(-1, d)[at]
            if k.shape[0]:
                out[u] = torch.softmax(q[u] @ k.t(), -1) @ v
        return {"out": out.view(c["batch"], c["hq"], d)}
    u, at, row = _rows_of(s)
    h = u % c["hkv"]
    hh = h if c["fused"] else h * 0                          # the head's place in the dense tensor that is written
    page = s["table"].view(units, -1)[u, at // p].long()
    got = {}
    if c["op"] == "read":
        for name, keys in (("K", True), ("V", False)):
            got[name + "_back"] = s[name + "_back"].double().contiguous()
            got[name + "_back"][row, hh] = _stored(c, s[name + "_pages"], keys)[page, at % p]
        return got
    turn = lambda x, rows: x                                 # noqa: E731
    if c["axes"]:
        def turn(x, rows):
            cos, sin = _angles(s, rows, torch.float64)
            z = torch.complex(x[..., :d // 2], x[..., d // 2:]) * torch.complex(cos, sin)[:, None]
            return torch.cat((z.real, z.imag), -1)
    k = turn(s["K"][row, h].double()[:, None], row)[:, 0]
    if c["fmt"] == "rows":
        for name, x in (("K", k), ("V", s["V"][row, h].double())):
            got[name + "_pages"] = s[name + "_pages"].double()
            got[name + "_pages"][page, at % p] = x
    else:
        # the stored row is the rotated one in the rows' type; a step to the next code either way is as near
        for name, x in (("K", k.to(_dtype(c)).double()), ("V", s["V"][row, h].double())):
            lo, hi = x.view(-1, d // 32, 32).amin(-1, True), x.view(-1, d // 32, 32).amax(-1, True)
            step = ((hi - lo) * 16 / 15).half().double()
            base = (lo - step).half().double()
            code = (16 * (x.view(-1, d // 32, 32) - base) / step - 16).round().clamp(0, 15)
            got[name + "_back"] = s[name + "_back"].double().contiguous()
            got[name + "_back"][row, hh] = (base + step * (1 + code / 16)).view(-1, d)
    if c["bounds"]:
        kept = s["K_bounds"].double()
        for sign, i in ((1, 0), (-1, 1)):
            x = torch.full((s["n_pages"], p, d), math.inf, dtype=torch.float64, device=DEV)
            x[page, at % p] = sign * k
            old = sign * s["K_bounds"][:, i].double()
            old[page[at % p == 0]] = math.inf
            low = torch.minimum(x.amin(1), old)
            kept[:, i] = torch.where(torch.isinf(low), kept[:, i], sign * low)
        got["K_bounds"] = kept
    if c["fused"]:
        n = s["Q"].shape[0] - c["pad"]
        got["Q_out"] = s["Q_out"].double()
        got["Q_out"][:n] = turn(s["Q"][:n].double(), torch.arange(n, device=DEV))
    return got

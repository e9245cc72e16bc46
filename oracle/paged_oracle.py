"""Float64 statement of the operators on a paged cache (numpy, one head at a time; test infrastructure only).

Pages are the bytes of the library's format (include/mixkv.h); every function below works on one layer.  Bf16 arrays are uint16 bit
patterns inside pages and float64 values outside.
"""
from __future__ import annotations

import numpy as np


def bf16_bits(x):
    """float64 -> bf16 bit patterns, by way of fp32, to nearest even."""
    u = np.ascontiguousarray(x, dtype=np.float64).astype(np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def as_dtype(x, dtype):
    """The values that the dtype holds, float64."""
    if dtype == "f32":
        return np.asarray(x, np.float64).astype(np.float32).astype(np.float64)
    return (bf16_bits(x).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


# ---- rotation
def axis_of_pairs(half, sections):
    return np.zeros(half, int) if sections is None else np.repeat(np.arange(3), sections)


def rotate(x, cos, sin, positions, sections, dtype):
    """One row x [D]; positions: one number per axis.  The pair (x_i, x_{i + D/2}) turns by the angle of its axis's position."""
    half = len(x) // 2
    at = np.clip(np.asarray(positions, np.int64)[axis_of_pairs(half, sections)], 0, len(cos) - 1)
    c, s = cos[at, np.arange(half)].astype(np.float64), sin[at, np.arange(half)].astype(np.float64)
    a, b = x[:half], x[half:]
    return as_dtype(np.concatenate([a * c - b * s, b * c + a * s]), dtype)


# ---- 4 bits
def quantise(row):
    """(codes [D], steps [D/32], bases [D/32]) of one row."""
    g = np.clip(row, -16384.0, 16384.0).reshape(-1, 32)
    lo, hi = g.min(1), g.max(1)
    step = ((hi - lo) * (16.0 / 15.0)).astype(np.float32).astype(np.float16)
    base = ((lo - step.astype(np.float64)).astype(np.float32) + np.float32(0)).astype(np.float16)      # no negative zero
    s, b = step.astype(np.float64)[:, None], base.astype(np.float64)[:, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        code = np.where(s > 0, np.clip(np.rint((g - b - s) * 16.0 / s), 0, 15), 0)
    return code.astype(int).reshape(-1), step, base


def element(code, step, base):
    """B + S (1 + code / 16), as fp32 arithmetic gives it."""
    return (base.astype(np.float64) + step.astype(np.float64) * (1.0 + code / 16.0)).astype(np.float32).astype(np.float64)


def nibble(e):
    return e // 2 + 4 * (e % 2)


def page_bytes(fmt, dtype, P, D):
    return P * D * 5 // 8 if fmt == "4bit" else P * D * (2 if dtype == "bf16" else 4)


def places(keys, r, d, D):
    """Where element d of row r lies in a 4-bit page of P rows: (word, nibble, fp16 of S, fp16 of B), counted from the codes' and the
    scales' beginning."""
    g = d // 32
    if keys:
        order = [0, 2, 1, 3] if D == 128 else [0, 1]
        word, e = r * (D // 8) + (d % 32) // 8 * (D // 32) + order[g], d % 8
        at = 2 * (r * (D // 32) + order[g])
        return word, nibble(e), at, at + 1
    t, q = r // 32, r % 16 // 4
    e = 2 * (r % 4) + (r % 32) // 16
    word = (4 * t + q) * D + d // 64 * 64 + 4 * (d % 16) + d % 64 // 16
    at = ((4 * t + q) * (D // 32) + g) * 16 + e
    return word, nibble(e), at, at + 8


class _Places:
    """places() of a whole page as arrays."""
    _kept = {}

    def __new__(cls, keys, P, D):
        if (keys, P, D) not in cls._kept:
            cls._kept[keys, P, D] = np.array([[places(keys, r, d, D) for d in range(D)] for r in range(P)])
        return cls._kept[keys, P, D]


def write_row(page, fmt, dtype, keys, P, r, row):
    """Row r of a page (uint8 array, in place)."""
    D = len(row)
    if fmt == "rows":
        raw = bf16_bits(row).view(np.uint8) if dtype == "bf16" else row.astype(np.float32).view(np.uint8)
        page[r * len(raw):(r + 1) * len(raw)] = raw
        return
    code, step, base = quantise(row)
    words, halves = page[:P * D // 2].view(np.uint32), page[P * D // 2:].view(np.float16)
    at = _Places(keys, P, D)[r]
    for d in range(D):
        w, n, s, b = at[d]
        words[w] = (int(words[w]) & ~(15 << (4 * n)) & 0xFFFFFFFF) | (int(code[d]) << (4 * n))
        halves[s], halves[b] = step[d // 32], base[d // 32]


def read_rows(page, fmt, dtype, keys, P, D):
    """All rows of a page, float64 [P, D] (4-bit elements in fp32)."""
    if fmt == "rows":
        if dtype == "f32":
            return page.view(np.float32).astype(np.float64).reshape(P, D)
        return (page.view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64).reshape(P, D)
    words, halves = page[:P * D // 2].view(np.uint32), page[P * D // 2:].view(np.float16)
    at = _Places(keys, P, D)
    code = (words[at[..., 0]] >> (4 * at[..., 1]).astype(np.uint32)) & 15
    with np.errstate(invalid="ignore", over="ignore"):
        return element(code.astype(np.float64), halves[at[..., 2]], halves[at[..., 3]])


# ---- the operators, on numpy copies of a layer's buffers
def _page(table, b, h, i, n_pages):
    return table[b, h, i] if 0 <= i < table.shape[2] and 0 <= table[b, h, i] < n_pages else -1


def append(fmt, dtype, P, D, K_pages, V_pages, bounds, table, lengths, K, V, row_start, row_count, Q=None, Q_out=None, rope=None):
    """In place.  K, V [n_rows, Hkv, D], Q [n_rows, Hq, D] float64 values; pages uint8 [n_pages, bytes]; bounds, Q_out float64.
    rope: (cos, sin, positions [axes, n_rows], sections or None)."""
    n_rows = K.shape[0]
    turn = (lambda x, r: x) if rope is None else (lambda x, r: rotate(x, rope[0], rope[1], rope[2][:, r], rope[3], dtype))
    for b, h in np.ndindex(*lengths.shape):
        n = min(max(int(lengths[b, h]), 0), table.shape[2] * P)
        count, start = max(int(row_count[b, h]), 0), int(row_start[b, h])
        for t in range(max(0, count - n, -start), min(count, n_rows - start)):
            r, src = n - count + t, start + t
            if Q is not None:
                G = Q.shape[1] // lengths.shape[1]
                for g in range(h * G, (h + 1) * G):
                    Q_out[src, g] = turn(Q[src, g], src)
            page = _page(table, b, h, r // P, len(K_pages))
            if page < 0:
                continue
            k = turn(K[src, h], src)
            write_row(K_pages[page], fmt, dtype, True, P, r % P, k)
            write_row(V_pages[page], fmt, dtype, False, P, r % P, V[src, h])
            if bounds is not None:
                if r % P == 0:
                    bounds[page] = k
                else:
                    bounds[page, 0], bounds[page, 1] = np.minimum(bounds[page, 0], k), np.maximum(bounds[page, 1], k)


def head(fmt, dtype, P, D, K_pages, V_pages, table, lengths, b, h, places_=None):
    """Keys and values of a head's rows, all or those of the listed places."""
    n = min(max(int(lengths[b, h]), 0), table.shape[2] * P)
    ks, vs = [np.zeros((0, D))], [np.zeros((0, D))]
    for i in (range(-(-n // P)) if places_ is None else places_):
        page = _page(table, b, h, int(i), len(K_pages))
        live = min(P, n - int(i) * P)
        if page < 0 or live <= 0:
            continue
        ks.append(read_rows(K_pages[page], fmt, dtype, True, P, D)[:live])
        vs.append(read_rows(V_pages[page], fmt, dtype, False, P, D)[:live])
    return np.concatenate(ks), np.concatenate(vs)


def read(fmt, dtype, P, D, K_pages, V_pages, table, lengths, K, V, row_start, row_count):
    """In place: dense rows K, V [n_rows, Hkv, D] (float64)."""
    for b, h in np.ndindex(*lengths.shape):
        n = min(max(int(lengths[b, h]), 0), table.shape[2] * P)
        count, start, pages = max(int(row_count[b, h]), 0), int(row_start[b, h]), {}
        for t in range(max(0, count - n, -start), min(count, K.shape[0] - start)):
            r, dst = n - count + t, start + t
            page = _page(table, b, h, r // P, len(K_pages))
            if page < 0:
                continue
            if page not in pages:
                pages[page] = [as_dtype(read_rows(x[page], fmt, dtype, keys, P, D), dtype) for x, keys in ((K_pages, True), (V_pages, False))]
            K[dst, h], V[dst, h] = (x[r % P] for x in pages[page])


def page_scores(Q, bounds, table, lengths, P, b, h):
    """fp32 scores of a head's pages, Q [batch, Hq, D]; a place without a page comes last."""
    G = Q.shape[1] // lengths.shape[1]
    q = Q[b, h * G:(h + 1) * G]
    up, down = np.maximum(q, 0).sum(0), np.minimum(q, 0).sum(0)
    n = min(max(int(lengths[b, h]), 0), table.shape[2] * P)
    out = np.full(-(-n // P), -np.inf, np.float32)
    known = {}
    for i in range(len(out)):
        page = _page(table, b, h, i, len(bounds))
        if page >= 0:
            if page not in known:
                hi, lo = np.where(up != 0, bounds[page, 1], 0.0), np.where(down != 0, bounds[page, 0], 0.0)
                known[page] = np.float32((hi * up + lo * down).sum())
            out[i] = known[page]
    return out


def select(scores, keep, first, last):
    """Places of the selected pages of one head, ascending."""
    n = len(scores)
    if n <= keep:
        return list(range(n))
    forced = set(range(first)) | set(range(n - last, n))
    rest = sorted((i for i in range(n) if i not in forced), key=lambda i: (-scores[i], i))
    return sorted(forced | set(rest[:keep - len(forced)]))


def attention(Q, k, v, scale):
    """One head's queries [G, D] over its rows."""
    if len(k) == 0:
        return np.zeros_like(Q)
    x = scale * (Q @ k.T)
    top = x.max(1, keepdims=True)
    if not np.isfinite(top).all():
        top = np.where(np.isneginf(top), 0.0, top)
    w = np.exp(x - top)
    total = w.sum(1, keepdims=True)
    return np.where(total > 0, (w @ v) / np.where(total > 0, total, 1.0), 0.0)


# ---- queries of new rows within a window, the weights they give, eviction by them
def sees(place, n, window, first):
    """Which of the places 0 ... n - 1 a row at `place` sees."""
    j = np.arange(n)
    return (j <= place) & ((j > place - window) | (j < first))


def rows_of(fmt, dtype, P, D, K_pages, V_pages, table, lengths, b, h):
    """Keys and values of a head by place, and which of the places have a page."""
    n = min(max(int(lengths[b, h]), 0), table.shape[2] * P)
    k, v, there = np.zeros((n, D)), np.zeros((n, D)), np.zeros(n, bool)
    for i in range(-(-n // P)):
        page, live = _page(table, b, h, i, len(K_pages)), min(P, n - i * P)
        if page >= 0:
            at = slice(i * P, i * P + live)
            k[at], v[at] = (read_rows(x[page], fmt, dtype, keys, P, D)[:live] for x, keys in ((K_pages, True), (V_pages, False)))
            there[at] = True
    return k, v, there


def new_rows(lengths, row_start, row_count, b, h, n, n_rows, max_count):
    """(row among the queries, place) of a head's new rows that are served."""
    count, start = max(int(row_count[b, h]), 0), int(row_start[b, h])
    return [(start + t, n - count + t) for t in range(min(count, max_count)) if 0 <= start + t < n_rows]


def window_attention(args, table, lengths, Q, row_start, row_count, window, first, max_count, scale, out, lse):
    """In place: out [n_rows, Hq, D], lse [n_rows, Hq] float64.  args: format, dtype, P, D and the pools."""
    G = Q.shape[1] // lengths.shape[1]
    for b, h in np.ndindex(*lengths.shape):
        k, v, there = rows_of(*args, table, lengths, b, h)
        for row, place in new_rows(lengths, row_start, row_count, b, h, len(k), len(Q), max_count):
            at = sees(place, len(k), window, first) & there
            heads = slice(h * G, (h + 1) * G)
            x = scale * (Q[row, heads] @ k[at].T)
            out[row, heads] = attention(Q[row, heads], k[at], v[at], scale)
            top = x.max(1, initial=-np.inf)
            safe = np.where(np.isneginf(top), 0.0, top)
            with np.errstate(divide="ignore"):
                lse[row, heads] = safe + np.log(np.exp(x - safe[:, None]).sum(1))


def window_weights(args, table, lengths, Q, row_start, row_count, window, first, max_count, scale, lse, weights):
    """In place: weights [n_pages, P] float64."""
    P = args[2]
    G = Q.shape[1] // lengths.shape[1]
    for b, h in np.ndindex(*lengths.shape):
        k, _, there = rows_of(*args, table, lengths, b, h)
        got = np.zeros(len(k))
        for row, place in new_rows(lengths, row_start, row_count, b, h, len(k), len(Q), max_count):
            at = sees(place, len(k), window, first) & there
            for g in range(h * G, (h + 1) * G):
                if not np.isneginf(lse[row, g]):
                    got[at] += np.exp(scale * (k[at] @ Q[row, g]) - lse[row, g])
        for j in np.nonzero(there)[0]:
            page = table[b, h, j // P]
            weights[page, j % P] = (0.0 if j >= len(k) - max(int(row_count[b, h]), 0) else weights[page, j % P]) + got[j]


def evicted(weights, there, keep, first, last):
    """Places of one head that are kept, ascending; weights and there by place."""
    n = len(weights)
    x = np.where(np.isnan(weights), -np.inf, weights)
    x[np.arange(n) < first] = np.inf
    x[np.arange(n) >= n - last] = np.inf
    best = sorted((j for j in range(n) if there[j]), key=lambda j: (-x[j], j))
    return sorted(best[:max(keep, 0)])


def evict(args, table, lengths, into, weights, weights_into, keep, max_keep, first, last, K_into, V_into, bounds_into):
    """In place: the pools (uint8) and weights that the rows go to, bounds [n_pages, 2, D] or None.  Returns (kept, n_kept)."""
    fmt, dtype, P, D, K, V = args
    kept, n_kept = np.full(lengths.shape + (max_keep,), -1, np.int32), np.zeros(lengths.shape, np.int32)
    for b, h in np.ndindex(*lengths.shape):
        n = min(max(int(lengths[b, h]), 0), table.shape[2] * P)
        there = np.array([_page(table, b, h, j // P, len(K)) >= 0 for j in range(n)], bool)
        w = np.array([weights[table[b, h, j // P], j % P] if there[j] else 0.0 for j in range(n)])
        at = evicted(w, there, min(int(keep[b, h]), max_keep), first, last)
        kept[b, h, :len(at)], n_kept[b, h] = at, len(at)
        for i, j in enumerate(at):
            src, dst = table[b, h, j // P], _page(into, b, h, i // P, len(K_into))
            if dst < 0:
                continue
            if weights_into is not None:
                weights_into[dst, i % P] = w[j]
            for pool, to, keys in ((K, K_into, True), (V, V_into, False)):
                move_row(pool[src], j % P, to[dst], i % P, fmt, dtype, keys, P, D)
            if bounds_into is not None:
                row = as_dtype(read_rows(K[src], fmt, dtype, True, P, D)[j % P], dtype)
                bounds_into[dst] = row if i % P == 0 else [np.minimum(bounds_into[dst, 0], row), np.maximum(bounds_into[dst, 1], row)]
    return kept, n_kept


def move_row(src, r, dst, i, fmt, dtype, keys, P, D):
    """Row r of one page becomes row i of another, bit for bit."""
    if fmt == "rows":
        w = D * (2 if dtype == "bf16" else 4)
        dst[i * w:(i + 1) * w] = src[r * w:(r + 1) * w]
        return
    a, z = _Places(keys, P, D)[r], _Places(keys, P, D)[i]
    sw, dw = src[:P * D // 2].view(np.uint32), dst[:P * D // 2].view(np.uint32)
    sh, dh = src[P * D // 2:].view(np.uint16), dst[P * D // 2:].view(np.uint16)
    for d in range(D):
        code = int(sw[a[d, 0]]) >> int(4 * a[d, 1]) & 15
        dw[z[d, 0]] = int(dw[z[d, 0]]) & ~(15 << int(4 * z[d, 1])) & 0xFFFFFFFF | code << int(4 * z[d, 1])
        dh[z[d, 2]], dh[z[d, 3]] = sh[a[d, 2]], sh[a[d, 3]]

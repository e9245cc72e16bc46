"""mixkv_paged_window_attention and mixkv_paged_weights against the float64 oracle: tolerances in tests/newrows.py."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2510_20707_amd import binding as B
from tests import newrows as R
from tests import paged as T

pytestmark = pytest.mark.gpu
KINDS = [("rows", "f32"), ("rows", "bf16"), ("4bit", "bf16")]


def _weights_too(rng, rows, q, window=R.ALL, first=0, scale=1.0, max_count=None, max_rows=None, cache=None):
    lay = rows.lay
    before = rng.random((lay.n_pages, lay.P)).astype(np.float32)
    w = torch.from_numpy(before.copy()).to(T.DEV)
    B.mixkv_paged_weights(lay.params(rows.hq, scale), [cache or lay.device()], [q], [w], window, first, max_count=max_count or rows.max_count, max_rows=max_rows)
    got = w.cpu().numpy()
    R.check_weights(rows, q.lse.cpu().numpy(), before, got, window, first, scale, max_count)
    return got


def _both(rng, rows, window=R.ALL, first=0, scale=1.0, max_count=None, max_rows=None, strided=False):
    q = R.attend(rows, window, first, scale, max_count, max_rows, strided)
    R.check_attention(rows, q, window, first, scale, max_count)
    _weights_too(rng, rows, q, window, first, scale, max_count, max_rows)
    return q


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P,G", [(128, 64, 7), (64, 32, 4), (128, 32, 16), (64, 128, 1), (128, 128, 17)])
@pytest.mark.parametrize("window,first", [(R.ALL, 0), (1, 0), (40, 3), (64, 33)])
def test_single_tokens(fmt, dtype, D, P, G, window, first):
    print(f"[case] one {fmt} {dtype} D={D} P={P} G={G} window={window} first={first}", flush=True)
    rng = np.random.default_rng([61, D, P, G])
    lens = np.array([[1, 2, 31], [32, 33, P], [P + 1, 2 * P - 1, 0], [127, 128, 129], [257, 96, 160]])
    lay = T.Layer(rng, fmt, dtype, D, P, lens, 9, fill=True)
    rows = R.Rows(rng, lay, 3 * G, np.ones(5))
    a = _both(rng, rows, window, first)
    b = _both(rng, rows, window, first, max_rows=300)
    assert torch.equal(b.out, R.attend(rows, window, first, max_rows=300).out)       # repeated bit for bit
    _both(rng, rows, window, first, max_rows=1)                                      # longer than the host said
    assert (a.out[2, 2 * G:] == 0).all() and torch.isneginf(a.lse[2, 2 * G:]).all() and (a.out[5:] == 7).all() and (a.lse[5:] == 7).all()


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P,G,counts", [(128, 64, 7, [5, 1, 0, 9]), (64, 32, 4, [17, 16, 15, 1]), (128, 32, 1, [33, 2, 64, 31]), (64, 128, 20, [3, 2, 1, 0])])
@pytest.mark.parametrize("window,first", [(R.ALL, 0), (1, 0), (30, 2), (100, 70), (7, 200)])
def test_a_few_rows(fmt, dtype, D, P, G, counts, window, first):
    print(f"[case] few {fmt} {dtype} D={D} P={P} G={G} window={window} first={first}", flush=True)
    rng = np.random.default_rng([62, D, P, G])
    lens = np.array([[5, 130], [300, 17], [64, 33], [97, 250]])
    lay = T.Layer(rng, fmt, dtype, D, P, lens, -(-300 // P), fill=True)
    rows = R.Rows(rng, lay, 2 * G, np.minimum(np.array(counts)[:, None], lens))      # (heads of fewer rows than the sequence has)
    _both(rng, rows, window, first, strided=True)
    _both(rng, rows, window, first, scale=0.3, max_rows=100)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P,G", [(128, 64, 7), (64, 32, 4), (128, 128, 1), (64, 64, 12)])
@pytest.mark.parametrize("window,first", [(R.ALL, 0), (1, 0), (70, 5), (150, 40), (33, 300)])
def test_prompts(fmt, dtype, D, P, G, window, first):
    """Whole prompts, chunks behind rows of before, and a sequence without rows, in one call."""
    print(f"[case] prompts {fmt} {dtype} D={D} P={P} G={G} window={window} first={first}", flush=True)
    rng = np.random.default_rng([63, D, P, G])
    lens = np.array([[321, 321], [40, 40], [0, 0], [500, 433]])
    lay = T.Layer(rng, fmt, dtype, D, P, lens, -(-500 // P) + 1, fill=True)
    rows = R.Rows(rng, lay, 2 * G, [321, 40, 0, 130])
    a = _both(rng, rows, window, first)
    assert torch.equal(a.out, R.attend(rows, window, first).out)
    assert (a.out[-3:] == 7).all() and (a.lse[-3:] == 7).all()
    _both(rng, rows, window, first, max_rows=64, strided=True)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,G", [(128, 2), (64, 7)])
def test_a_chunk_behind_a_long_cache(fmt, dtype, D, G):
    """Few groups of rows, many tiles: the tiles of a group go to several workgroups."""
    print(f"[case] long {fmt} {dtype} D={D} G={G}", flush=True)
    rng = np.random.default_rng([64, D])
    P = 128
    lay = T.Layer(rng, fmt, dtype, D, P, [[2900, 1500]], 23, fill=True)
    for count in (1, 6, 100):
        rows = R.Rows(rng, lay, 2 * G, [count])
        for window, first in ((R.ALL, 0), (1400, 130)):
            q = _both(rng, rows, window, first)
            assert torch.equal(q.out, R.attend(rows, window, first).out) and torch.equal(q.lse, R.attend(rows, window, first).lse)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("count", [1, 6, 400])
def test_heads_longer_than_the_host_said(fmt, dtype, count):
    rng = np.random.default_rng([74, count])
    lay = T.Layer(rng, fmt, dtype, 64, 64, [[1800, 900]], 29, fill=True)
    rows = R.Rows(rng, lay, 8, [count])
    for window, first in ((R.ALL, 0), (700, 40)):
        _both(rng, rows, window, first, max_rows=300)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,G,count", [(128, 33, 1), (64, 80, 1), (64, 130, 2), (128, 257, 1)])
def test_more_query_heads_than_a_group(fmt, dtype, D, G, count):
    rng = np.random.default_rng([75, G])
    lay = T.Layer(rng, fmt, dtype, D, 64, [[70, 300], [1, 129]], 5, fill=True)
    rows = R.Rows(rng, lay, 2 * G, [count] * 2)
    for window, first in ((R.ALL, 0), (50, 3)):
        _both(rng, rows, window, first, strided=True)


@pytest.mark.parametrize("fmt,dtype", [("rows", "bf16"), ("4bit", "bf16")])
@pytest.mark.parametrize("window,first", [(R.ALL, 0), (100, 600), (900, 10)])
def test_prompts_of_several_blocks_and_chunks(fmt, dtype, window, first):
    """More keys than a workgroup takes, more rows than a chunk has, first rows that fill a block."""
    print(f"[case] blocks {fmt} window={window} first={first}", flush=True)
    rng = np.random.default_rng([76, first])
    lay = T.Layer(rng, fmt, dtype, 64, 128, [[1500, 700]], 12, fill=True)
    rows = R.Rows(rng, lay, 6, np.array([[1500, 700]]))
    q = _both(rng, rows, window, first)
    w = [torch.zeros((lay.n_pages, lay.P), device=T.DEV) for _ in range(2)]
    for x in w:
        B.mixkv_paged_weights(lay.params(rows.hq), [lay.device()], [q], [x], window, first)
    assert torch.equal(*w)                                                           # repeated bit for bit


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("count", [1, 4, 90])
def test_rows_and_pages_that_are_none(fmt, dtype, count):
    """Entries that are no page, lengths beyond the table and below zero, more new rows than the head has, rows outside the dense ones, more than max_count."""
    rng = np.random.default_rng([65, count])
    D, P = 64, 32
    lay = T.Layer(rng, fmt, dtype, D, P, [[150, 200], [1000, -5], [60, 61]], 8, fill=True)
    lay.table[0, 0, 1], lay.table[0, 1, 0], lay.table[0, 1, 5] = lay.n_pages, -7, 2 ** 31 - 1
    lay.table[1, 0, 7] = -1                                                          # the new row's own page
    rows = R.Rows(rng, lay, 6, [count] * 3)
    rows.start[0, 1], rows.start[2] = -2, rows.n - 2                                 # rows before the first one, and behind the last
    rows.start[1, 1] = 2 ** 31 - 1
    rows.count[2, 1] = 2 ** 31 - 1                                                   # most of them before the head's first row
    q = _both(rng, rows, max_count=count)
    assert torch.isfinite(q.out.float()).all()
    _both(rng, rows, 20, 3, max_count=count)
    if count > 1:
        _both(rng, rows, 20, 3, max_count=count - 1)
    rows.count[1] = -3
    _both(rng, rows, max_count=count)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P", [(128, 64), (64, 32)])
@pytest.mark.parametrize("counts", [[1, 1], [6, 3], [150, 120]])
def test_what_is_not_seen_may_be_anything(fmt, dtype, D, P, counts):
    """NaN and infinities behind the last row, and (full precision) in keys and values that the window leaves out, or that only the newest rows see."""
    rng = np.random.default_rng([66, D, counts[0]])
    lens = np.array([[200, 170], [151, 130]])
    lay = T.Layer(rng, fmt, dtype, D, P, lens, -(-200 // P), fill=True)
    window, first = 20, 5
    odd = np.array([np.nan, np.inf, -np.inf])
    for b, h in np.ndindex(2, 2):
        n = int(lens[b, h])
        for pool, keys in ((lay.K, True), (lay.V, False)):
            for r in range(n, -(-n // P) * P):                                       # rows that do not exist
                page = pool[lay.table[b, h, r // P]]
                if fmt == "rows":
                    O.write_row(page, fmt, dtype, keys, P, r % P, odd[np.arange(D) % 3])
                else:
                    halves, at = page[P * D // 2:].view(np.uint16), O._Places(keys, P, D)[r % P]
                    halves[at[:, 2]], halves[at[:, 3]] = 0x7E00, 0xFC00
            if fmt == "rows":
                out_of_sight = [j for j in (first, first + 1, n - counts[b] - window) if j >= first] if counts[b] < 100 else []
                for j in out_of_sight:
                    O.write_row(pool[lay.table[b, h, j // P]], fmt, dtype, keys, P, j % P, odd[np.arange(D) % 3])
    rows = R.Rows(rng, lay, 6, counts)
    q = _both(rng, rows, window, first)
    assert torch.isfinite(q.out[:sum(counts)].float()).all()
    if fmt == "4bit":
        return
    # the values of a row near the end: an infinity in one element, a NaN in another; only the rows that see it have them
    for b, h in np.ndindex(2, 2):
        for j in (lens[b, h] - 1, lens[b, h] - 1 - counts[b] // 2):
            page = lay.V[lay.table[b, h, j // P]]
            row = O.read_rows(page, fmt, dtype, False, P, D)[j % P]
            row[3], row[D - 2] = np.inf, np.nan
            O.write_row(page, fmt, dtype, False, P, j % P, row)
    q = R.attend(rows, window, first)
    out, _ = R.check_attention(rows, q, window, first)
    assert np.isinf(out[:, :, 3]).any() and (counts[0] == 1 or np.isfinite(out[0]).all())


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("count", [1, 5, 80])
@pytest.mark.parametrize("spread,scale", [(60.0, 1.0), (2.0, 30.0), (1e-4, 1.0)])
def test_logits_far_apart_and_near_each_other(fmt, dtype, count, spread, scale):
    rng = np.random.default_rng([67, count, int(spread)])
    lay = T.Layer(rng, fmt, dtype, 128, 32, [[300, 290]], 10, fill=True)
    rows = R.Rows(rng, lay, 6, [count], spread=spread)
    for window, first in ((R.ALL, 0), (50, 10)):
        q = R.attend(rows, window, first, scale)
        R.check_attention(rows, q, window, first, scale)
        if spread < 60:
            _weights_too(rng, rows, q, window, first, scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count", [1, 5, 80])
def test_rows_of_no_weight(dtype, count):
    """Keys of minus infinity: whole tiles, whole windows."""
    rng = np.random.default_rng([68, count])
    D, P, n = 128, 32, 300
    lay = T.Layer(rng, "rows", dtype, D, P, [[n]], 10, fill=True)
    rows = R.Rows(rng, lay, 5, [count])
    rows.Q[..., 7] = O.as_dtype(np.abs(rows.Q[..., 7]) + 0.5, dtype)
    for off in (np.arange(n) // 32 % 3 != 1, np.arange(n) < n - 3, np.ones(n, bool)):
        for r in range(n):
            page = lay.table[0, 0, r // P]
            row = O.read_rows(lay.K[page], "rows", dtype, True, P, D)[r % P]
            row[7] = -np.inf if off[r] else 0.25
            O.write_row(lay.K[page], "rows", dtype, True, P, r % P, row)
        for window, first in ((R.ALL, 0), (40, 20)):
            q = R.attend(rows, window, first)
            out, lse = np.full(rows.Q.shape, 7.0), np.full(rows.Q.shape[:2], 7.0)
            finite = T.Layer.args(lay)
            with np.errstate(invalid="ignore", over="ignore"):
                O.window_attention(finite, lay.table, lay.lengths, rows.Q, rows.start, rows.count, window, first, rows.max_count, 1.0, out, lse)
            got = T.values(q.out)
            assert np.isfinite(got).all() and np.array_equal(np.isneginf(q.lse.cpu().numpy()), np.isneginf(lse))
            v = max(np.abs(O.rows_of(*lay.args(), lay.table, lay.lengths, 0, 0)[1]).max(), 1.0)
            assert (np.abs(got - out) <= 2.0 ** -6 * v).all() and (got[np.isneginf(lse)] == 0).all()


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_rows_see_the_same_whatever_the_kernel(fmt, dtype):
    """A prompt's rows one at a time, a few at a time and together: the same up to the roundings."""
    rng = np.random.default_rng(69)
    lay = T.Layer(rng, fmt, dtype, 64, 32, [[140, 140]], 5, fill=True)
    rows = R.Rows(rng, lay, 6, [140], pad=0)
    whole = R.attend(rows, 33, 4)
    R.check_attention(rows, whole, 33, 4)
    one = R.Rows(rng, lay, 6, [1], pad=0)
    for t in (0, 31, 32, 36, 37, 139):
        lay.lengths[:] = t + 1
        one.Q = rows.Q[t:t + 1]
        q = R.attend(one, 33, 4)
        R.check_attention(one, q, 33, 4)
        assert (q.out.float() - whole.out[t:t + 1].float()).abs().max() <= 2.0 ** -5 * 4
        assert (q.lse - whole.lse[t:t + 1]).abs().max() <= 1e-2 if fmt == "4bit" else 1e-4


def test_without_lse_and_with_many_layers():
    """More layers than a launch takes, each with buffers of its own; no lse asked for."""
    rng = np.random.default_rng(70)
    layers = [T.Layer(rng, "rows", "bf16", 64, 32, [[50 + i, 40]], 3, fill=True) for i in range(35)]
    n_pages = max(l.n_pages for l in layers)
    for count in (1, 50):
        qs, caches, rows = [], [], []
        for lay in layers:
            rows.append(R.Rows(rng, lay, 4, [min(count, 40)]))
            qs.append(rows[-1].device())
            qs[-1].lse = None
            c = lay.device()
            grow = lambda t: torch.cat((t, t[:1].expand(n_pages - t.shape[0], *t.shape[1:]))).contiguous()  # noqa: E731
            caches.append(B.PagedCache(grow(c.K_pages), grow(c.V_pages), c.page_table, c.lengths))
        p = layers[0].params(4)
        p.n_pages = n_pages
        B.mixkv_paged_window_attention(p, caches, qs, 20, 2, max_count=count)
        for lay, r, q in zip(layers, rows, qs):
            out, lse = np.full(r.Q.shape, 7.0), np.full(r.Q.shape[:2], 7.0)
            O.window_attention(*r.args(), 20, 2, count, 1.0, out, lse)
            assert np.abs(T.values(q.out) - out).max() <= 2.0 ** -7 * 5 + 1e-3
        w = [torch.ones((n_pages, 32), device=T.DEV) for _ in layers]
        for q, r in zip(qs, rows):
            lse = np.full(r.Q.shape[:2], 7.0)
            O.window_attention(*r.args(), 20, 2, count, 1.0, np.zeros(r.Q.shape), lse)
            q.lse = torch.from_numpy(lse).float().to(T.DEV)
        B.mixkv_paged_weights(p, caches, qs, w, 20, 2, max_count=count)
        for lay, r, q, x in zip(layers, rows, qs, w):
            R.check_weights(r, q.lse.cpu().numpy(), np.ones((lay.n_pages, 32), np.float32), x[:lay.n_pages].cpu().numpy(), 20, 2, max_count=count)


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_lse_is_what_the_compression_asks_for(fmt, dtype):
    """The whole path: a prompt appended with its rotation, its causal attention with the log-sum-exp, weights, eviction, the next token's rows and attention within a
    window; and mixkv_compress on the rows read back takes the log-sum-exp of the last rows and keeps what it keeps without."""
    rng = np.random.default_rng(71)
    D, P, hkv, G, n, W = 64, 32, 2, 3, 200, 8
    lay = T.Layer(rng, fmt, dtype, D, P, [[n + 1, n + 1]], 8, spare=9, fill=False)
    lay.lengths[:] = n
    cache, p, hq = lay.device(), lay.params(hkv * G, 0.125), hkv * G
    angle = rng.random((300, D // 2)) * 6
    cos, sin = (torch.from_numpy(f(angle).astype(np.float32)).to(T.DEV) for f in (np.cos, np.sin))
    dt = B.TORCH_DTYPE[p.dtype]
    new = lambda m: [torch.from_numpy(rng.standard_normal((m, x, D)) + 0.3).to(T.DEV).to(dt) for x in (hkv, hkv, hq)]  # noqa: E731
    K, V, Q = new(n)
    start, count = T.i32(np.zeros((1, hkv))), T.i32(np.full((1, hkv), n))
    q_out = torch.empty_like(Q)
    B.mixkv_paged_append(p, [cache], [B.PagedRows(K, V, start, count, Q, q_out)], B.Rope(cos, sin, torch.arange(n, dtype=torch.int32, device=T.DEV)[None]))
    lay.K, lay.V = cache.K_pages.cpu().numpy().view(np.uint8).reshape(lay.K.shape), cache.V_pages.cpu().numpy().view(np.uint8).reshape(lay.V.shape)
    rows = R.Rows(rng, lay, hq, [n], pad=0)
    rows.Q = T.values(q_out)
    q = B.PagedQueries(q_out, start, count, torch.empty_like(q_out), torch.empty((n, hq), device=T.DEV))
    B.mixkv_paged_window_attention(p, [cache], [q], max_count=n)
    R.check_attention(rows, q, scale=0.125)
    # the compression, with and without it
    dense = B.PagedRows(torch.empty_like(K), torch.empty_like(V), start, count)
    B.mixkv_paged_read(p, [cache], [dense], max_count=n)
    Kd, Vd = (t.permute(1, 0, 2)[None].contiguous() for t in (dense.K, dense.V))
    cp = B.make_params(dtype, 1, hq, hkv, D, n, W, 40, causal_window=True, softmax_scale=0.125)
    Qw = q_out[-W:].permute(1, 0, 2)[None].contiguous()
    lse = q.lse[-W:].t()[None].contiguous()
    scores = []
    for given in (None, [lse]):
        out = B.alloc_layer_out(cp, T.DEV)
        B.mixkv_compress(cp, [Kd], [Vd], [Qw], [out], B.alloc_workspace(cp, 1, T.DEV), window_lse=given)
        scores.append(out.scores[..., :n - W].cpu().numpy())
    assert np.abs(scores[1] - scores[0]).max() <= 2e-2 * np.abs(scores[0]).max()     # (4-bit elements are rounded to bf16 on their way back)
    # weights, eviction to 60 rows, the next token within a window
    w = torch.zeros((lay.n_pages, P), device=T.DEV)
    B.mixkv_paged_weights(p, [cache], [q], [w], max_count=n)
    R.check_weights(rows, q.lse.cpu().numpy(), np.zeros((lay.n_pages, P), np.float32), w.cpu().numpy(), scale=0.125)
    total = sum(float(w[lay.table[0, h, :7], :].flatten()[:n].sum()) for h in range(hkv))
    assert abs(total - n * hq) <= 1e-2 * n * hq                                       # every row gives one
    free = [i for i in range(lay.n_pages) if i not in set(lay.table.flatten().tolist())]
    into = B.PagedCache(cache.K_pages, cache.V_pages, T.i32(np.array([[free[:4] + [-1] * 4, free[4:8] + [-1] * 4]])), T.i32(np.zeros((1, hkv))))
    (kept,) = B.mixkv_paged_evict(p, [cache], [into], [w], [T.i32(np.full((1, hkv), 60))], 60, 4, 16, weights_into=[w])
    weights = w.cpu().numpy()
    for h in range(hkv):
        at = np.array([weights[lay.table[0, h, j // P], j % P] for j in range(n)])
        assert kept[0, h].tolist() == O.evicted(at, np.ones(n, bool), 60, 4, 16)
    assert into.lengths.tolist() == [[60, 60]]
    into.lengths.add_(1)
    K1, V1, Q1 = new(1)
    one = torch.empty_like(Q1)
    ones = T.i32(np.ones((1, hkv)))
    B.mixkv_paged_append(p, [into], [B.PagedRows(K1, V1, start, ones, Q1, one)], B.Rope(cos, sin, torch.full((1, 1), n, dtype=torch.int32, device=T.DEV)))
    lay.K, lay.V = into.K_pages.cpu().numpy().view(np.uint8).reshape(lay.K.shape), into.V_pages.cpu().numpy().view(np.uint8).reshape(lay.V.shape)
    lay.table, lay.lengths = into.page_table.cpu().numpy(), into.lengths.cpu().numpy()
    step = R.Rows(rng, lay, hq, [1], pad=0)
    step.Q = T.values(one)
    q1 = B.PagedQueries(one, start, ones, torch.empty_like(one), torch.empty((1, hq), device=T.DEV))
    B.mixkv_paged_window_attention(p, [into], [q1], 32, 4)
    R.check_attention(step, q1, 32, 4, 0.125)
    before = w.cpu().numpy()
    B.mixkv_paged_weights(p, [into], [q1], [w], 32, 4)
    R.check_weights(step, q1.lse.cpu().numpy(), before, w.cpu().numpy(), 32, 4, 0.125)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("count", [1, 3, 70])
def test_captured_and_on_another_stream(fmt, dtype, count):
    """Attention and weights captured into a graph on a side stream: replays with new queries and eager work between them give what the eager calls give."""
    rng = np.random.default_rng([72, count])
    lay = T.Layer(rng, fmt, dtype, 128, 64, [[700, 650], [300, 90]], 12, fill=True)
    cache, p = lay.device(), lay.params(6)
    rows = [R.Rows(rng, lay, 6, [count, min(count, 90)]) for _ in range(4)]
    q, other = rows[0].device(), rows[0].device()
    w, w2 = (torch.zeros((lay.n_pages, 64), device=T.DEV) for _ in range(2))
    att, wei = (B.PreparedPagedWindowAttention(p, [cache], [q], 200, 8, max_count=rows[0].max_count),
                B.PreparedPagedWeights(p, [cache], [q], [w], 200, 8, max_count=rows[0].max_count))
    att2, wei2 = (B.PreparedPagedWindowAttention(p, [cache], [other], 200, 8, max_count=rows[0].max_count),
                  B.PreparedPagedWeights(p, [cache], [other], [w2], 200, 8, max_count=rows[0].max_count))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        att.run(), wei.run()
    side.synchronize()
    w.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        att.run()
        wei.run()
    torch.cuda.synchronize()
    for r in rows:
        for x in (q, other):
            x.Q.copy_(T.to_device(r.Q, dtype))
        att2.run(), wei2.run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q.out, other.out) and torch.equal(q.lse, other.lse) and torch.equal(w, w2)
        assert float(torch.ones(1000, device=T.DEV).sum()) == 1000.0


@pytest.mark.parametrize("count", [1, 100])
def test_pools_beyond_four_gigabytes(count):
    """Page addresses and rows of queries that pass 32 bits."""
    D, P, n_pages, hq = 128, 128, 150000, 2
    rng = np.random.default_rng([73, count])
    n = 300
    K, V = (torch.empty((n_pages, P, D), dtype=torch.bfloat16, device=T.DEV) for _ in range(2))
    assert K.numel() * 2 > 2 ** 32
    ids = np.array([n_pages - 1, 5, n_pages - 77])
    small = T.Layer(rng, "rows", "bf16", D, P, [[n]], 3, spare=0, fill=True)
    for i in range(3):
        for pool, src in ((K, small.K), (V, small.V)):
            pool[ids[i]] = torch.from_numpy(src[small.table[0, 0, i]].view(np.int16).copy()).view(torch.bfloat16).view(P, D).to(T.DEV)
    p = B.make_paged_params("bf16", "rows", 1, hq, 1, D, P, 3, n_pages)
    cache = B.PagedCache(K, V, T.i32(ids[None, None]), T.i32([[n]]))
    rows = R.Rows(rng, small, hq, [count])
    q = rows.device()
    B.mixkv_paged_window_attention(p, [cache], [q], 120, 3, max_count=count)
    R.check_attention(rows, q, 120, 3)
    w = torch.zeros((n_pages, P), device=T.DEV)
    B.mixkv_paged_weights(p, [cache], [q], [w], 120, 3, max_count=count)
    got = np.zeros((3, P), np.float32)
    for i in range(3):
        got[small.table[0, 0, i]] = w[ids[i]].cpu().numpy()
    R.check_weights(rows, q.lse.cpu().numpy(), np.zeros((3, P), np.float32), got, 120, 3)
    assert float(w.double().sum()) == pytest.approx(float(got.astype(np.float64).sum()), rel=1e-6)

"""mixkv_paged_select and mixkv_paged_attention against the float64 oracle.

Selections are compared exactly: both sides form the scores in 64 bits and rank their fp32 roundings (two orders of the sum differ
by 2^-45 of its terms, so that a rounding, 2^-24 of the score, is decided otherwise in one score of some 10^5 where terms cancel
tenfold; the scores here are equal or 2^-20 apart).

Attention, per output row (one query head): |gpu - oracle| <= tol * max_d |oracle_d|.
  f32    1e-5: fp32 accumulation over at most a few thousand rows, as in mixkv_decode_attention.
  bf16   2^-8 + 1e-4, as there: the output's rounding, 2^-8 of the element, and the fp32 sums before it.
  4bit   2^-8 + 1e-4 + 2 * 2^-11 * max_j |v_j| / max |out|: beside those, values and weights enter the second product in fp16, each
         rounded by at most 2^-11 of itself, so that sum_j w_j v_j moves by at most 2 * 2^-11 * sum_j w_j |v_j| <= 2 * 2^-11 * max |v|."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2510_20707_amd import binding as B
from tests import paged as T

pytestmark = pytest.mark.gpu
KINDS = [("rows", "f32"), ("rows", "bf16"), ("4bit", "bf16")]
TOL = {"f32": 1e-5, "bf16": 2.0 ** -8 + 1e-4}


def _queries(rng, lay, hq, spread=2.0):
    return O.as_dtype(rng.standard_normal((lay.lengths.shape[0], hq, lay.D)) * spread / np.sqrt(lay.D), lay.dtype)


def _attend_and_check(lay, Q, scale=1.0, lists=None, max_rows=None, logit_error=0.0):
    """lists[b][h]: places of the selected pages.  logit_error d: weights off by a factor e^+-d move the output by 2 d max |v|."""
    hq = Q.shape[1]
    G = hq // lay.lengths.shape[1]
    cache = lay.device()
    args = {}
    if lists is not None:
        most = max(max((len(x) for row in lists for x in row), default=1), 1)
        sel = np.full(lay.lengths.shape + (most,), -5, np.int32)
        n = np.zeros(lay.lengths.shape, np.int32)
        for b, h in np.ndindex(*lay.lengths.shape):
            n[b, h] = len(lists[b][h])
            sel[b, h, :n[b, h]] = lists[b][h]
        args = dict(selected=[T.i32(sel)], n_selected=[T.i32(n)])
    got = T.values(B.mixkv_paged_attention(lay.params(hq, scale), [cache], [T.to_device(Q, lay.dtype)], max_rows=max_rows, **args)[0])
    worst = 0.0
    for b, h in np.ndindex(*lay.lengths.shape):
        k, v = O.head(*lay.args(), lay.table, lay.lengths, b, h, None if lists is None else lists[b][h])
        want = O.attention(Q[b, h * G:(h + 1) * G], k, v, scale)
        for g in range(G):
            err, top = np.abs(got[b, h * G + g] - want[g]).max(), np.abs(want[g]).max()
            limit = TOL[lay.dtype] * top + ((2 * 2.0 ** -11 * (lay.fmt == "4bit") + 2 * logit_error) * np.abs(v).max() if len(v) else 0.0)
            assert err <= limit, f"b{b} h{h} g{g}, {len(k)} rows: {err:.3e} over {limit:.3e}"
            worst = max(worst, err / limit if limit else 0.0)
    print(f"       {worst:.3f} of the tolerance", flush=True)
    return got


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P,G", [(128, 64, 7), (64, 32, 4), (128, 32, 16), (64, 128, 1), (128, 128, 17), (64, 64, 40)])
def test_lengths_around_tiles_pages_and_waves(fmt, dtype, D, P, G):
    print(f"[case] attention {fmt} {dtype} D={D} P={P} G={G}", flush=True)
    rng = np.random.default_rng([11, D, P, G])
    lens = np.array([[1, 2, 31], [32, 33, P], [P + 1, 2 * P - 1, 0], [127, 128, 129], [257, 96, 160]])
    lay = T.Layer(rng, fmt, dtype, D, P, lens, 9, fill=True)
    Q = _queries(rng, lay, 3 * G)
    a = _attend_and_check(lay, Q)
    b = _attend_and_check(lay, Q, max_rows=300)                    # several chunks of a head, and repeated bit for bit
    assert np.array_equal(b, _attend_and_check(lay, Q, max_rows=300))
    _attend_and_check(lay, Q, max_rows=1)                          # longer than the host said
    assert (a[2, 2 * G:] == 0).all()


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_long_heads_in_a_ragged_batch(fmt, dtype, D):
    P = 128
    print(f"[case] attention long {fmt} {dtype} D={D}", flush=True)
    rng = np.random.default_rng([12, D])
    lay = T.Layer(rng, fmt, dtype, D, P, [[2600, 0], [5, 700]], 21, fill=True)
    Q = _queries(rng, lay, 12)
    _attend_and_check(lay, Q)
    _attend_and_check(lay, Q, max_rows=1000)
    _attend_and_check(lay, Q, scale=0.37)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("spread,scale", [(60.0, 1.0), (2.0, 30.0), (1e-4, 1.0), (500.0, 3.0)])
def test_logits_far_apart_and_near_each_other(fmt, dtype, spread, scale):
    # the largest logit comes late, early, anywhere; with the steepest the softmax picks one row.  A logit is a fp32 sum of D terms, off by
    # at most D 2^-24 of their magnitudes' sum; 4-bit keys are summed as S sum(q u) + B sum(q) with u in [1, 2), whose terms are up to
    # 2 S + |B| <= 8 max |k| times |q|: S <= 2.2 max |k|, |B| <= 3.2 max |k|
    rng = np.random.default_rng([13, int(spread), int(scale)])
    D, P = 128, 32
    lay = T.Layer(rng, fmt, dtype, D, P, [[300, 90]], 10, fill=True)
    Q = _queries(rng, lay, 6, spread)
    terms = 0.0
    for h in range(2):
        k, _ = O.head(*lay.args(), lay.table, lay.lengths, 0, h)
        if fmt == "4bit":
            terms = max(terms, float(np.abs(Q[0, 3 * h:3 * h + 3]).sum(1).max() * 8 * np.abs(k).max()))
        else:
            terms = max(terms, float((np.abs(Q[0, 3 * h:3 * h + 3]) @ np.abs(k).T).max()))
    _attend_and_check(lay, Q, scale=scale, logit_error=D * 2.0 ** -24 * terms * scale)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P", [(128, 64), (64, 32)])
def test_selected_pages(fmt, dtype, D, P):
    print(f"[case] attention selected {fmt} {dtype} D={D} P={P}", flush=True)
    rng = np.random.default_rng([14, D, P])
    lens = np.array([[7 * P + 3, 5 * P], [2 * P - 1, 0], [P, 6 * P + 31]])
    lay = T.Layer(rng, fmt, dtype, D, P, lens, 9, fill=True)
    Q = _queries(rng, lay, 10)
    _attend_and_check(lay, Q, lists=[[[0, 3, 7], [1]], [[1], []], [[0], [2, 4, 5, 6]]])
    # any order, the newest page not among them, places without rows, a page twice, places that are none in the table, an empty list
    _attend_and_check(lay, Q, lists=[[[6, 0, 2, 8], [4, 4, 0]], [[0, -1, 9, 2 ** 31 - 1, -2 ** 31], [0, 1]], [[], [6]]])
    _attend_and_check(lay, Q, lists=[[list(range(8)), [3, 1, 2]], [[1, 0], []], [[8], [0]]], max_rows=1)


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_pages_that_do_not_exist_have_no_rows(fmt, dtype):
    rng = np.random.default_rng(15)
    D, P = 128, 32
    lay = T.Layer(rng, fmt, dtype, D, P, [[100, 200], [1000, -5]], 8, fill=True)      # longer than the table: as long as it
    lay.table[0, 0, 1], lay.table[0, 1, 0], lay.table[0, 1, 5] = lay.n_pages, -7, 2 ** 31 - 1
    lay.table[1, 0, :] = -1
    Q = _queries(rng, lay, 4)
    got = _attend_and_check(lay, Q)
    assert (got[1] == 0).all()
    _attend_and_check(lay, Q, lists=[[[1, 2], [0, 1, 5]], [[3], [0]]])


def _poison(lay):
    """Rows that do not exist, in pages that do: everything in them a NaN or an infinity."""
    for pool, keys in ((lay.K, True), (lay.V, False)):
        for b, h in np.ndindex(*lay.lengths.shape):
            n = int(lay.lengths[b, h])
            for r in range(n, -(-n // lay.P) * lay.P):
                page = pool[lay.table[b, h, r // lay.P]]
                if lay.fmt == "rows":
                    w = 2 if lay.dtype == "bf16" else 4
                    raw = np.array([0x7FC0, 0xFF80, 0x7F80], np.uint16)[np.arange(lay.D) % 3].astype(np.uint32)
                    page[r % lay.P * lay.D * w:(r % lay.P + 1) * lay.D * w] = (raw.astype(np.uint16) if w == 2 else raw << 16).view(np.uint8)
                else:
                    halves = page[lay.P * lay.D // 2:].view(np.uint16)
                    at = O._Places(keys, lay.P, lay.D)[r % lay.P]
                    halves[at[:, 2]], halves[at[:, 3]] = 0x7E00, 0xFC00


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P", [(128, 64), (64, 128)])
def test_nan_and_infinities_behind_the_last_row(fmt, dtype, D, P):
    rng = np.random.default_rng([16, D])
    lay = T.Layer(rng, fmt, dtype, D, P, [[1, 33, 70], [P - 1, 2 * P + 5, 31]], 4, fill=True)
    _poison(lay)
    Q = _queries(rng, lay, 6)
    got = _attend_and_check(lay, Q)
    assert np.isfinite(got).all()
    _attend_and_check(lay, Q, lists=[[[0], [0], list(range(-(-70 // P)))], [[0], [2, 0], [0]]])


@pytest.mark.parametrize("fmt,dtype", [("rows", "f32"), ("rows", "bf16")])
@pytest.mark.parametrize("masked", ["scattered", "tiles", "front", "all but one", "all"])
def test_rows_of_no_weight(fmt, dtype, masked):
    rng = np.random.default_rng(17)
    D, P, n = 128, 32, 300
    lay = T.Layer(rng, fmt, dtype, D, P, [[n]], 10, fill=True)
    off = {"scattered": rng.random(n) < 0.3, "tiles": np.arange(n) // 32 % 4 != 2, "front": np.arange(n) < n - 3, "all but one": np.arange(n) != n - 5,
           "all": np.ones(n, bool)}[masked]
    Q = _queries(rng, lay, 5)
    Q[..., 7] = O.as_dtype(np.abs(Q[..., 7]) + 0.5, dtype)
    for r in np.nonzero(off)[0]:
        page = lay.table[0, 0, r // P]
        row = O.read_rows(lay.K[page], fmt, dtype, True, P, D)[r % P]
        row[7] = -np.inf
        O.write_row(lay.K[page], fmt, dtype, True, P, r % P, row)
    for most in (None, 256):
        got = _attend_and_check(lay, Q, max_rows=most)
        assert np.isfinite(got).all() and (masked != "all" or (got == 0).all())


@pytest.mark.parametrize("value", [3e-5, 1e-7, 60000.0, 0.0])
def test_4bit_values_tiny_and_large(value):
    rng = np.random.default_rng(18)
    D, P = 128, 32
    lay = T.Layer(rng, "4bit", "bf16", D, P, [[200]], 7, fill=True)
    for r in range(200):
        O.write_row(lay.V[lay.table[0, 0, r // P]], "4bit", "bf16", False, P, r % P, O.as_dtype(rng.standard_normal(D) * min(value, 4000.0), "bf16"))
    # fp16 resolves 2^-25 below its normal numbers: an element B + S u is rounded by that too
    Q, lim = _queries(rng, lay, 4), 2.0 ** -24
    got = T.values(B.mixkv_paged_attention(lay.params(4), [lay.device()], [T.to_device(Q, "bf16")])[0])
    k, v = O.head(*lay.args(), lay.table, lay.lengths, 0, 0)
    want = O.attention(Q[0], k, v, 1.0)
    assert (np.abs(got[0] - want) <= (2.0 ** -8 + 1e-4) * np.abs(want).max(1, keepdims=True) + 2.0 ** -10 * np.abs(v).max() + lim).all()


# ---- selection
def _select_and_check(lay, Q, keep, first, last):
    most_pages = lay.table.shape[2]
    (sel,), (n,) = B.mixkv_paged_select(lay.params(Q.shape[1]), [lay.device()], [T.to_device(Q, lay.dtype)], keep, first, last)
    sel, n = sel.cpu().numpy(), n.cpu().numpy()
    for b, h in np.ndindex(*lay.lengths.shape):
        s = O.page_scores(Q, lay.bounds, lay.table, lay.lengths, lay.P, b, h)
        assert len(s) <= most_pages
        want = O.select(s, keep, first, last)
        assert n[b, h] == len(want) and sel[b, h].tolist() == want + [-1] * (keep - len(want)), (b, h, len(s))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,P,G", [(128, 32, 7), (64, 64, 1), (128, 64, 20)])
def test_selection(dtype, D, P, G):
    print(f"[case] select {dtype} D={D} P={P} G={G}", flush=True)
    rng = np.random.default_rng([19, D, G])
    lens = np.array([[300 * P, 7, 0], [P * 40 + 1, P * 8, P * 9], [P * 257, P * 600 - 3, P]])
    lay = T.Layer(rng, "rows", dtype, D, P, lens, 601, spare=0, bounds=True)
    lay.table[2, 1, 100:110] = -1
    lay.bounds.sort(axis=1)
    lay.K, lay.V = lay.K[:1], lay.V[:1]
    cache = lay.device
    lay.device = lambda: B.PagedCache(None, None, *(lambda c: (c.page_table, c.lengths, c.K_bounds))(cache()))
    Q = _queries(rng, lay, 3 * G)
    for keep, first, last in ((8, 1, 1), (1, 0, 0), (64, 4, 2), (3, 2, 1), (5, 0, 5), (256, 1, 1), (700, 1, 1)):
        _select_and_check(lay, Q, keep, first, last)


@pytest.mark.parametrize("what", ["equal", "two values", "zeros of both signs", "infinite", "negative"])
def test_selection_of_equal_scores(what):
    rng = np.random.default_rng(20)
    D, P, n = 64, 32, 500
    lay = T.Layer(rng, "4bit", "bf16", D, P, [[n * P, n * P - 40]], n, spare=0, bounds=True)
    Q = np.ones((1, 2, D))
    v = {"equal": np.full(lay.n_pages, 2.0), "two values": rng.integers(0, 2, lay.n_pages) + 1.0, "zeros of both signs": np.where(rng.random(lay.n_pages) < 0.5, 0.0, -0.0),
         "infinite": np.where(rng.random(lay.n_pages) < 0.3, -np.inf, np.where(rng.random(lay.n_pages) < 0.01, np.inf, 1.0)),
         "negative": -rng.integers(1, 5, lay.n_pages).astype(float)}[what]
    lay.bounds = np.zeros((lay.n_pages, 2, D))
    lay.bounds[:, :, 3] = v[:, None]
    Q[:, :, :3] = Q[:, :, 4:] = 0.0
    lay_scores = lay.bounds[:, 1, 3] * 2.0                               # two queries of 1 there and 0 elsewhere
    for keep in (3, 17, 250, 499):
        (sel,), _ = B.mixkv_paged_select(lay.params(4), [lay.device()], [T.to_device(np.repeat(Q, 2, 1), "bf16")], keep, 1, 1)
        for h in range(2):
            s = lay_scores[lay.table[0, h, :n - h]]                      # the second head is a page shorter
            assert np.array_equal(O.page_scores(np.repeat(Q, 2, 1), lay.bounds, lay.table, lay.lengths, P, 0, h), s.astype(np.float32))
            assert sel[0, h].tolist() == O.select(s, keep, 1, 1), (keep, h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pages", [500, 3000, 17000])
def test_pages_whose_score_is_nan_come_last(dtype, pages):
    D, P = 64, 32
    rng = np.random.default_rng([23, pages])
    lay = T.Layer(rng, "rows", dtype, D, P, [[pages * P]], pages, spare=0, bounds=True)
    lay.K, lay.V = lay.K[:1], lay.V[:1]
    cache = lay.device()
    bad = rng.random(pages) < 0.5                                        # by place in the table
    bits = cache.K_bounds.view(torch.int32 if dtype == "f32" else torch.int16)
    ids = cache.page_table[0, 0, :pages].long()
    bits[ids[torch.from_numpy(bad).to(ids.device)], 0, 5] = -1           # all bits of a smallest key set: a NaN of negative sign
    Q = np.full((1, 1, D), -1.0)
    good = int((~bad).sum())
    for keep in (good - 3, good + 20):
        (sel,), (n,) = B.mixkv_paged_select(lay.params(1), [B.PagedCache(None, None, cache.page_table, cache.lengths, cache.K_bounds)],
                                            [T.to_device(Q, dtype)], keep, 0, 0)
        got = sel[0, 0].cpu().numpy()
        assert n.item() == keep and np.all(np.diff(got) > 0) and got[0] >= 0 and got[-1] < pages
        taken = np.zeros(pages, bool)
        taken[got] = True
        if keep < good:
            assert not np.any(taken & bad)
        else:                                                            # the earliest ones of them
            assert np.all(taken[~bad]) and np.array_equal(np.flatnonzero(taken & bad), np.flatnonzero(bad)[:keep - good])


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_a_decoding_loop(fmt, dtype):
    """A prompt, then eight tokens: rotated rows appended, pages selected, attention over those and over all, against the oracle's own
    cache; everything on a stream of its own."""
    rng = np.random.default_rng(21)
    D, P, hkv, G, batch, prompt, steps = 64, 32, 2, 3, 2, np.array([150, 61]), 8
    lay = T.Layer(rng, fmt, dtype, D, P, np.repeat((prompt + steps)[:, None], hkv, 1), 6, bounds=True)
    lay.lengths[:] = 0
    cache, p, hq = lay.device(), lay.params(hkv * G, 0.125), hkv * G
    angle = rng.random((300, D // 2)) * 6
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    cosd, sind = (torch.from_numpy(x).to(T.DEV) for x in (cos, sin))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def step(counts, check):
        n = int(counts.sum())
        K, V, Q = (O.as_dtype(rng.standard_normal((n, h, D)) + 0.3, dtype) for h in (hkv, hkv, hq))
        pos = np.concatenate([l + np.arange(c) for l, c in zip(lay.lengths[:, 0], counts)]).astype(np.int32)[None]
        start = np.repeat((np.cumsum(counts) - counts)[:, None], hkv, 1)
        count = np.repeat(counts[:, None], hkv, 1)
        lay.lengths += count.astype(np.int32)
        want_q = np.zeros(Q.shape)
        O.append(*lay.args(), lay.bounds, lay.table, lay.lengths, K, V, start, count, Q, want_q, (cos, sin, pos, None))
        with torch.cuda.stream(side):
            cache.lengths.add_(T.i32(count))
            q_out = torch.zeros(Q.shape, dtype=B.TORCH_DTYPE[p.dtype], device=T.DEV)
            rows = B.PagedRows(T.to_device(K, dtype), T.to_device(V, dtype), T.i32(start), T.i32(count), T.to_device(Q, dtype), q_out)
            B.mixkv_paged_append(p, [cache], [rows], B.Rope(cosd, sind, T.i32(pos)))
            if not check:
                side.synchronize()
                return
            (sel,), (n_sel,) = B.mixkv_paged_select(p, [cache], [q_out], 3)
            dense = B.mixkv_paged_attention(p, [cache], [q_out])[0]
            few = B.mixkv_paged_attention(p, [cache], [q_out], [sel], [n_sel])[0]
        side.synchronize()
        assert np.array_equal(T.values(q_out), want_q) and np.array_equal(cache.K_pages.cpu().numpy(), lay.K)
        assert np.array_equal(cache.V_pages.cpu().numpy(), lay.V)
        for b, h in np.ndindex(batch, hkv):
            s = O.page_scores(want_q, lay.bounds, lay.table, lay.lengths, P, b, h)
            chosen = O.select(s, 3, 1, 1)
            assert sel[b, h, :len(chosen)].tolist() == chosen and n_sel[b, h] == len(chosen)
            for got, places in ((dense, None), (few, chosen)):
                k, v = O.head(*lay.args(), lay.table, lay.lengths, b, h, places)
                want = O.attention(want_q[b, h * G:(h + 1) * G], k, v, p.softmax_scale)
                err = np.abs(T.values(got)[b, h * G:(h + 1) * G] - want).max(1)
                assert (err <= TOL[dtype] * np.abs(want).max(1) + (2.0 ** -10 * np.abs(v).max() if fmt == "4bit" else 0)).all()

    step(prompt, False)
    for _ in range(steps):
        step(np.array([1, 1]), True)


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_a_captured_step_replays(fmt, dtype):
    """A decoding step (lengths advanced, rows appended, pages selected, attention) captured once: every replay, with new rows in the same
    buffers and eager work in between, gives what the eager calls give on a cache of their own, bit for bit."""
    rng = np.random.default_rng(22)
    D, P, hkv, hq, batch = 128, 32, 2, 8, 3
    lay = T.Layer(rng, fmt, dtype, D, P, np.repeat([[300], [70], [33]], hkv, 1), 12, spare=10, bounds=True, fill=True)
    lay.lengths -= 8
    caches, p = [lay.device(), lay.device()], lay.params(hq, 0.1)
    dt = B.TORCH_DTYPE[p.dtype]
    new = lambda *shape: torch.zeros(shape, dtype=dt, device=T.DEV)  # noqa: E731
    one, start = torch.ones((batch, hkv), dtype=torch.int32, device=T.DEV), T.i32(np.repeat(np.arange(batch)[:, None], hkv, 1))
    K, V, Q, pos = new(batch, hkv, D), new(batch, hkv, D), new(batch, hq, D), torch.zeros((1, batch), dtype=torch.int32, device=T.DEV)
    angle = torch.rand((500, D // 2), device=T.DEV) * 6
    rope = B.Rope(angle.cos(), angle.sin(), pos)
    sides = []
    for c in caches:
        q_out, out, few = new(batch, hq, D), new(batch, hq, D), new(batch, hq, D)
        sel, n_sel = torch.zeros((batch, hkv, 4), dtype=torch.int32, device=T.DEV), torch.zeros((batch, hkv), dtype=torch.int32, device=T.DEV)
        calls = (B.PreparedPagedAppend(p, [c], [B.PagedRows(K, V, start, one, Q, q_out)], rope, max_count=1),
                 B.PreparedPagedSelect(p, [c], [q_out], [sel], [n_sel]), B.PreparedPagedAttention(p, [c], [q_out], [out]),
                 B.PreparedPagedAttention(p, [c], [q_out], [few], [sel], [n_sel]))
        sides.append((c, calls, (q_out, out, few, sel, n_sel)))

    def step(c, calls):
        c.lengths.add_(one)
        for call in calls:
            call.run()

    def fill():
        for t in (K, V, Q):
            t.copy_(torch.from_numpy(rng.standard_normal(tuple(t.shape))).to(dt))
        pos.copy_(torch.from_numpy(rng.integers(0, 500, (1, batch)).astype(np.int32)))

    fill()
    step(*sides[0][:2])                                               # as a program warms up, on both caches
    step(*sides[1][:2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*sides[1][:2])
    for _ in range(4):
        fill()
        step(*sides[0][:2])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(sides[0][2] + (caches[0].K_pages, caches[0].V_pages, caches[0].K_bounds), sides[1][2] + (caches[1].K_pages, caches[1].V_pages, caches[1].K_bounds)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        assert all(torch.isfinite(t.float()).all() for t in sides[0][2])


def test_python_refuses_what_the_pointers_do_not_say():
    rng = np.random.default_rng(23)
    lay = T.Layer(rng, "rows", "bf16", 64, 32, [[40, 40]], 2, bounds=True)
    c, p, q = lay.device(), lay.params(4), torch.zeros((1, 4, 64), dtype=torch.bfloat16, device=T.DEV)
    rows = lambda **kw: [B.PagedRows(**{**dict(K=torch.zeros((5, 2, 64), dtype=torch.bfloat16, device=T.DEV),  # noqa: E731
                                               V=torch.zeros((5, 2, 64), dtype=torch.bfloat16, device=T.DEV), row_start=T.i32([[0, 0]]), row_count=T.i32([[5, 5]])), **kw})]
    other = lambda **kw: B.PagedCache(**{**c.__dict__, **kw})  # noqa: E731
    for bad in (lambda: B.mixkv_paged_append(p, [c], rows(K=torch.zeros((5, 2, 64), device=T.DEV))),
                lambda: B.mixkv_paged_append(p, [c], rows(V=torch.zeros((5, 2, 64), dtype=torch.bfloat16))),
                lambda: B.mixkv_paged_append(p, [c], rows(V=torch.zeros((4, 2, 64), dtype=torch.bfloat16, device=T.DEV))),
                lambda: B.mixkv_paged_append(p, [c], rows(row_count=torch.zeros((1, 2), dtype=torch.int64, device=T.DEV))),
                lambda: B.mixkv_paged_append(p, [c], rows(Q=torch.zeros((5, 4, 64), dtype=torch.bfloat16, device=T.DEV))),
                lambda: B.mixkv_paged_append(p, [c], rows(), B.Rope(torch.zeros((9, 32), device=T.DEV), torch.zeros((8, 32), device=T.DEV), T.i32([[0] * 5]))),
                lambda: B.mixkv_paged_append(p, [c], rows(), B.Rope(torch.zeros((9, 32), device=T.DEV), torch.zeros((9, 32), device=T.DEV), T.i32([[0] * 5] * 3))),
                lambda: B.mixkv_paged_append(p, [c], rows(), B.Rope(torch.zeros((9, 32), device=T.DEV), torch.zeros((9, 32), device=T.DEV), T.i32([[0] * 4]))),
                lambda: B.mixkv_paged_read(p, [other(K_pages=c.K_pages[:-1])], rows()),
                lambda: B.mixkv_paged_attention(p, [other(page_table=c.page_table[..., :1])], [q]),
                lambda: B.mixkv_paged_attention(p, [c], [q.float()]),
                lambda: B.mixkv_paged_attention(p, [c], [q], [T.i32([[[0], [0]]])], [T.i32([[1]])]),
                lambda: B.mixkv_paged_select(p, [other(K_bounds=None)], [q], 2),
                lambda: B.mixkv_paged_select(p, [other(K_bounds=c.K_bounds.float())], [q], 2),
                lambda: B.mixkv_paged_attention(p, [other(lengths=c.lengths.cpu())], [q])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.mixkv_paged_select(p, [c], [q], 2, 2, 1), lambda: B.mixkv_paged_select(p, [c], [q], 2, workspace=None)):
        with pytest.raises(B.MixkvError) as e:
            bad()
        assert e.value.status == B.MIXKV_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("pages,distinct", [(1023, 1023), (1025, 40), (4100, 4100), (4096, 7), (16384, 3000), (16390, 500), (40001, 40001)])
def test_selection_among_many_pages(dtype, D, pages, distinct):
    # every kernel that ranks, with few and with many equal scores; a head of few pages beside the long one
    rng = np.random.default_rng([24, pages])
    P, G = 32, 3
    lay = T.Layer(rng, "rows", dtype, D, P, [[P, P]], pages, spare=distinct - 2, bounds=True)
    lay.lengths[0] = [pages * P - 5, 70]
    lay.table[0] = rng.integers(0, lay.n_pages, (2, pages))
    if pages < 5000:
        lay.table[0, 0, 17:30] = -1
    lay.bounds.sort(axis=1)
    Q = _queries(rng, lay, 2 * G)
    table, lengths, bounds = T.i32(lay.table), T.i32(lay.lengths), T.to_device(lay.bounds, dtype)
    cache = B.PagedCache(None, None, table, lengths, bounds)
    scores = [O.page_scores(Q, lay.bounds, lay.table, lay.lengths, P, 0, h) for h in range(2)]
    for keep, first, last in ((16, 1, 1), (1000, 3, 4), (pages - 1, 0, 1), (2, 1, 1)):
        (sel,), (n,) = B.mixkv_paged_select(lay.params(2 * G), [cache], [T.to_device(Q, dtype)], keep, first, last)
        for h in range(2):
            want = O.select(scores[h], keep, first, last)
            assert n[0, h] == len(want) and sel[0, h].tolist() == want + [-1] * (keep - len(want)), (keep, h)


@pytest.mark.parametrize("fmt,page_bytes", [("rows", 32768), ("4bit", 10240)])
def test_pages_and_rows_beyond_four_gigabytes(fmt, page_bytes):
    """The same rows through a small pool and at the end of one of more than 2^32 bytes, from the end of a dense tensor of more than 2^32
    bytes: every output agrees bit for bit."""
    D, P, n, batch = 128, 128, 300, 1
    far_pages, far_rows = (1 << 32) // page_bytes + 40, (1 << 32) // (2 * D) + 5000
    g = torch.Generator(device=T.DEV).manual_seed(25)
    K, V, Q = (torch.randn((n, 1, D), generator=g, device=T.DEV).bfloat16() for _ in range(3))
    angle = torch.rand((400, D // 2), generator=g, device=T.DEV) * 6
    pos = torch.randint(0, 400, (1, n), generator=g, device=T.DEV).int()
    got = []
    for pages, rows in ((8, n), (far_pages, far_rows)):
        p = B.make_paged_params("bf16", fmt, batch, 1, 1, D, P, 3, pages, 0.2)
        cache = B.alloc_paged_cache(p, T.DEV, bounds=True)
        assert pages == 8 or cache.K_pages.numel() * cache.K_pages.element_size() > 1 << 32
        cache.page_table[0, 0] = torch.arange(pages - 3, pages, device=T.DEV)
        cache.lengths.fill_(n)
        at = rows - n
        dense = [torch.empty((rows, 1, D), dtype=torch.bfloat16, device=T.DEV) for _ in range(4)]
        for t, x in zip(dense, (K, V, Q)):
            t[at:] = x
        where = torch.zeros((1, rows), dtype=torch.int32, device=T.DEV)
        where[:, at:] = pos
        one = lambda x: torch.full((1, 1), x, dtype=torch.int32, device=T.DEV)  # noqa: E731
        B.mixkv_paged_append(p, [cache], [B.PagedRows(dense[0], dense[1], one(at), one(n), dense[2], dense[3])], B.Rope(angle.cos(), angle.sin(), where), n)
        q = dense[3][-1:].contiguous().view(1, 1, D)
        dense[0][at:] = 0
        dense[1][at:] = 0
        B.mixkv_paged_read(p, [cache], [B.PagedRows(dense[0], dense[1], one(at), one(n))], n)
        (sel,), (m,) = B.mixkv_paged_select(p, [cache], [q], 2)
        outs = [t[at:].clone() for t in (dense[3], dense[0], dense[1])] + [sel, m, cache.K_bounds[pages - 3:].clone()]
        outs += [B.mixkv_paged_attention(p, [cache], [q])[0], B.mixkv_paged_attention(p, [cache], [q], [sel], [m])[0]]
        # a step of one row more, by the kernel for few rows
        cache.lengths.fill_(n + 1)
        B.mixkv_paged_append(p, [cache], [B.PagedRows(dense[3], dense[2], one(rows - 1), one(1), dense[2], torch.empty_like(dense[2]))], None, 1)
        outs += [cache.K_pages[pages - 3:].clone(), cache.V_pages[pages - 3:].clone()] if fmt == "rows" else []
        outs.append(B.mixkv_paged_attention(p, [cache], [q])[0])
        torch.cuda.synchronize()
        got.append([t.cpu() for t in outs])
        del dense, cache, outs
        torch.cuda.empty_cache()
    for a, b in zip(*got):
        live = a.shape == b.shape and torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
        # (rows of the last page that were never written are whatever the allocation held)
        if not live and a.dim() == 3 and a.shape[0] == 3 and fmt == "rows" and a.shape[1] == P:
            flat = lambda t: t.reshape(-1, D)[:n + 1].contiguous().view(torch.uint8)  # noqa: E731
            live = torch.equal(flat(a), flat(b))
        assert live


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_more_layers_than_one_launch_takes(fmt, dtype):
    D, P, L = 64, 32, 35
    rng = np.random.default_rng(26)
    lens = [np.array([[5 + 7 * l, 300 - 8 * l]]) for l in range(L)]
    lays = [T.Layer(rng, fmt, dtype, D, P, n, 10, spare=0, bounds=True, fill=True) for n in lens]
    most = max(l.n_pages for l in lays)
    for l in lays:                                                       # pools of one size
        pad = most - l.n_pages
        l.K, l.V = (np.concatenate([x, np.zeros((pad, x.shape[1]), np.uint8)]) for x in (l.K, l.V))
        l.bounds = np.sort(np.concatenate([l.bounds, np.zeros((pad, 2, D))]), axis=1)
        l.n_pages = most
    Qs = [_queries(rng, l, 6) for l in lays]
    p, caches, q = lays[0].params(6), [l.device() for l in lays], [T.to_device(x, dtype) for x in Qs]
    sel, n = B.mixkv_paged_select(p, caches, q, 4)
    outs = B.mixkv_paged_attention(p, caches, q), B.mixkv_paged_attention(p, caches, q, sel, n)
    for l, lay in enumerate(lays):
        for h in range(2):
            places = O.select(O.page_scores(Qs[l], lay.bounds, lay.table, lay.lengths, P, 0, h), 4, 1, 1)
            assert sel[l][0, h, :len(places)].tolist() == places and n[l][0, h] == len(places)
            for out, which in zip(outs, (None, places)):
                k, v = O.head(*lay.args(), lay.table, lay.lengths, 0, h, which)
                want = O.attention(Qs[l][0, 3 * h:3 * h + 3], k, v, 1.0)
                err = np.abs(T.values(out[l])[0, 3 * h:3 * h + 3] - want).max(1)
                assert (err <= TOL[dtype] * np.abs(want).max(1) + (2.0 ** -10 * np.abs(v).max() if fmt == "4bit" else 0)).all(), (l, h)


def test_calls_on_two_streams_with_workspaces_of_their_own():
    rng = np.random.default_rng(27)
    lays = [T.Layer(rng, fmt, "bf16", 128, 32, [[900, 30], [1, 400]], 30, fill=True, bounds=True) for fmt in ("4bit", "rows")]
    jobs = []
    for lay in lays:
        c, q, p = lay.device(), T.to_device(_queries(rng, lay, 8), "bf16"), lay.params(8)
        alone = B.mixkv_paged_attention(p, [c], [q])[0], B.mixkv_paged_select(p, [c], [q], 5)[0][0]
        out, sel, n = torch.empty_like(q), torch.empty((2, 2, 5), dtype=torch.int32, device=T.DEV), torch.empty((2, 2), dtype=torch.int32, device=T.DEV)
        jobs.append((torch.cuda.Stream(), (B.PreparedPagedAttention(p, [c], [q], [out]), B.PreparedPagedSelect(p, [c], [q], [sel], [n])), alone, (out, sel)))
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, calls, _, got in jobs:
            with torch.cuda.stream(stream):
                for t in got:
                    t.zero_()
            for call in calls:
                call.run(stream)
        torch.cuda.synchronize()
        for _, _, alone, got in jobs:
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(alone, got))


def test_a_call_on_a_stream_of_its_own_allocates_there():
    """Outputs and workspace of a call on another stream are that stream's: work that still runs on the current one does not share their memory."""
    rng = np.random.default_rng(28)
    lay = T.Layer(rng, "4bit", "bf16", 128, 32, [[700, 900], [30, 400]], 30, fill=True, bounds=True)
    c, q, p = lay.device(), T.to_device(_queries(rng, lay, 8), "bf16"), lay.params(8)
    want, (sel,), side = B.mixkv_paged_attention(p, [c], [q])[0], B.mixkv_paged_select(p, [c], [q], 5)[0], torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.zeros(1 << 26, device=T.DEV)
    for _ in range(5):
        for _ in range(4):
            busy.add_(1)
        trash = [torch.full((1 << n,), 127, dtype=torch.uint8, device=T.DEV) for n in range(9, 20)]
        del trash                                                        # free for the current stream, still to be written to there
        out = B.mixkv_paged_attention(p, [c], [q], stream=side)[0]
        picked = B.mixkv_paged_select(p, [c], [q], 5, stream=side)[0][0]
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(picked, sel)


def test_a_prepared_call_belongs_to_its_device(monkeypatch):
    rng = np.random.default_rng(29)
    lay = T.Layer(rng, "rows", "f32", 64, 32, [[40, 7]], 2, fill=True, bounds=True)
    c, q, p = lay.device(), torch.zeros((1, 2, 64), device=T.DEV), lay.params(2)
    call = B.PreparedPagedAttention(p, [c], [q], [torch.empty_like(q)])
    call.run()
    torch.cuda.synchronize()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)         # as a program that has gone on to another device
    with pytest.raises(ValueError):
        call.run()
    with pytest.raises(ValueError):
        B.PreparedPagedAttention(p, [c], [q], [torch.empty_like(q)])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size,scale", [(0.0, 1e-12), (0.0, 1e-40), (2.0 ** 125, 1.0), (2.0 ** 100, 2.0 ** -100), (2.0 ** -118, 2.0 ** 120)])
def test_4bit_scores_at_the_ends_of_the_exponents(D, size, scale):
    """Queries and softmax scales far from one whose logits are ordinary: queries of zero, queries that meet nothing but zeros in the keys, a size
    and a scale that make up for one another.  The heads end inside a tile, so rows that do not exist are among the scores."""
    rng = np.random.default_rng([40, D])
    P = 32
    lay = T.Layer(rng, "4bit", "bf16", D, P, [[40, 1], [33, 70]], 3, fill=True)
    Q = _queries(rng, lay, 6)
    if size == 2.0 ** 125:                                               # all of the queries in the first 32 elements, where the keys have zeros
        Q[..., 32:] = 0.0
        for b, h in np.ndindex(2, 2):
            for r in range(int(lay.lengths[b, h])):
                page = lay.K[lay.table[b, h, r // P]]
                row = O.as_dtype(rng.standard_normal(D), "bf16")
                row[:32] = 0.0
                O.write_row(page, "4bit", "bf16", True, P, r % P, row)
    got = _attend_and_check(lay, Q * size, scale=scale)
    assert np.isfinite(got).all()


def _terms(lay, Q):
    """The largest sum of the magnitudes of a logit's terms (4-bit keys: S sum(q u) + B sum(q) with u in [1, 2), up to 8 max |k| times |q|)."""
    G, most = Q.shape[1] // lay.lengths.shape[1], 0.0
    for b, h in np.ndindex(*lay.lengths.shape):
        q, k = np.abs(Q[b, h * G:(h + 1) * G]), np.abs(O.head(*lay.args(), lay.table, lay.lengths, b, h)[0])
        k = k[np.isfinite(k).all(1)]
        if len(k):
            most = max(most, float(q.sum(1).max() * 8 * k.max() if lay.fmt == "4bit" else (q @ k.T).max()))
    return most


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,size", [(64, 1e20), (128, 1e30)])
def test_large_values_behind_rising_logits(dtype, D, size):
    """Logits that rise by 40 powers of two from one of a wave's tiles to its next, twice, and large values: a weight is at most a power of two above
    the first tile's, times a value of 1e30 no infinity."""
    rng = np.random.default_rng([41, D])
    P, n = 32, 300
    lay = T.Layer(rng, "rows", dtype, D, P, [[n, n - 13]], 10, fill=True)
    Q = _queries(rng, lay, 4)
    Q[..., 0] = 1.0
    for h in range(2):
        for r in range(int(lay.lengths[0, h])):
            page = lay.table[0, h, r // P]
            row = O.read_rows(lay.K[page], "rows", dtype, True, P, D)[r % P]
            row[0] = 28.0 * (r // 128)                                   # tile t is wave t % 4's
            O.write_row(lay.K[page], "rows", dtype, True, P, r % P, row)
            O.write_row(lay.V[page], "rows", dtype, False, P, r % P, O.as_dtype(rng.standard_normal(D) * size, dtype))
    got = _attend_and_check(lay, Q, logit_error=D * 2.0 ** -24 * _terms(lay, Q))
    assert np.isfinite(got).all()
    print(f"[case] large values {dtype} D={D}", flush=True)


def _chunks_are_several(lay, hq, max_rows):
    rows = lay.table.shape[2] * lay.P if max_rows is None else max_rows
    assert B.mixkv_paged_attention_workspace_size(lay.params(hq), 1, rows) > 0


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P,G", [(128, 64, 7), (64, 32, 1), (128, 32, 19)])
def test_heads_of_several_chunks(fmt, dtype, D, P, G):
    """Lengths around the borders of chunks of 128 rows, and the last chunk longer than the others."""
    print(f"[case] attention chunks {fmt} {dtype} D={D} P={P} G={G}", flush=True)
    rng = np.random.default_rng([42, D, P, G])
    lay = T.Layer(rng, fmt, dtype, D, P, [[127, 128, 129], [640, 513, 0], [255, 1, 400]], 640 // P, fill=True)
    Q = _queries(rng, lay, 3 * G)
    for most in (None, 385, 500):
        _chunks_are_several(lay, 3 * G, most)
        got = _attend_and_check(lay, Q, max_rows=most)
        assert np.array_equal(got, _attend_and_check(lay, Q, max_rows=most)) and (got[1, 2 * G:] == 0).all()


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("gone", ["first", "last", "between", "all but one", "all"])
def test_chunks_without_rows_or_weight(fmt, dtype, gone):
    """Whole chunks whose pages do not exist, and in full precision whole chunks of keys of minus infinity: their partial results have no offset."""
    D, P, n = 128, 32, 620
    for masked in (False, True):
        if masked and fmt == "4bit":
            continue
        rng = np.random.default_rng(43)
        lay = T.Layer(rng, fmt, dtype, D, P, [[n, n]], 20, fill=True)
        Q = _queries(rng, lay, 6)
        Q[..., 7] = O.as_dtype(np.abs(Q[..., 7]) + 0.5, dtype)
        chunk = np.arange(20) // 4
        off = {"first": chunk < 2, "last": chunk >= 3, "between": (chunk == 1) | (chunk == 3), "all but one": chunk != 2, "all": chunk >= 0}[gone]
        if not masked:
            lay.table[0, 0, off] = -1
        else:
            for place in np.nonzero(off)[0]:
                for r in range(P):
                    row = O.read_rows(lay.K[lay.table[0, 0, place]], fmt, dtype, True, P, D)[r]
                    row[7] = -np.inf
                    O.write_row(lay.K[lay.table[0, 0, place]], fmt, dtype, True, P, r, row)
        for most in (None, 400):
            _chunks_are_several(lay, 6, most)
            got = _attend_and_check(lay, Q, max_rows=most)
            assert np.isfinite(got).all() and (gone != "all" or (got[0, :3] == 0).all())


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("spread,scale", [(60.0, 1.0), (2.0, 30.0), (500.0, 3.0)])
def test_chunks_with_logits_far_apart(fmt, dtype, spread, scale):
    rng = np.random.default_rng([44, int(spread)])
    lay = T.Layer(rng, fmt, dtype, 128, 32, [[640, 390]], 20, fill=True)
    Q = _queries(rng, lay, 6, spread)
    _chunks_are_several(lay, 6, None)
    _attend_and_check(lay, Q, scale=scale, logit_error=128 * 2.0 ** -24 * _terms(lay, Q) * scale)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_chunks_of_more_tiles_than_a_wave_has_lanes_for(fmt, dtype, D):
    """A wave asks for the table entries of 64 tiles at a time: heads of 9001 and 17 000 rows as one chunk each, all their pages and listed ones."""
    print(f"[case] attention long chunks {fmt} {dtype} D={D}", flush=True)
    rng = np.random.default_rng([45, D])
    P = 32
    lay = T.Layer(rng, fmt, dtype, D, P, [[8 * P, 8 * P]], 600, spare=0, fill=True)
    lay.table[:] = rng.integers(0, lay.n_pages, lay.table.shape)
    lay.table[0, :, 300:303] = -1
    lay.lengths[0] = 17000, 9001
    Q = _queries(rng, lay, 6)
    error = D * 2.0 ** -24 * _terms(lay, Q)
    _attend_and_check(lay, Q, max_rows=1, logit_error=error)
    _attend_and_check(lay, Q, max_rows=1, lists=[[rng.permutation(600).tolist(), rng.integers(0, 282, 600).tolist()]], logit_error=error)


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_more_chunks_than_a_workgroup_has_threads(fmt, dtype):
    """264 chunks of 16 tiles: the threads that fold them take a second one each."""
    print(f"[case] attention many chunks {fmt} {dtype}", flush=True)
    rng = np.random.default_rng(46)
    D, P, n = 64, 128, 135000
    lay = T.Layer(rng, fmt, dtype, D, P, [[16 * P]], -(-n // P), spare=0, fill=True)
    lay.table[:] = rng.integers(0, lay.n_pages, lay.table.shape)
    lay.lengths[0] = n
    Q = _queries(rng, lay, 3)
    p = lay.params(3)
    assert B.mixkv_paged_attention_workspace_size(p, 1, n) >= 257 * 3 * (D + 2) * 4
    _attend_and_check(lay, Q, logit_error=D * 2.0 ** -24 * _terms(lay, Q))
    lay.lengths[0] = 300                                                 # most of them without rows
    _attend_and_check(lay, Q, logit_error=D * 2.0 ** -24 * _terms(lay, Q))


@pytest.mark.parametrize("dtype,D,pages", [("bf16", 64, 600), ("bf16", 128, 600), ("f32", 64, 600), ("f32", 128, 600), ("f32", 128, 1200)])
def test_selection_in_several_steps(dtype, D, pages):
    """Many heads: a workgroup scores several steps of 32 to 128 pages, the last case more than the eight that it takes at most.  Heads end before, at
    and behind the borders of steps and of workgroups, and entries that are no page lie in all of them."""
    print(f"[case] select steps {dtype} D={D} pages={pages}", flush=True)
    rng = np.random.default_rng([47, D, pages])
    P, batch, hkv, G = 32, 64, 8, 2
    step = 4 * 8 * (64 // (2 * D * (2 if dtype == "bf16" else 4) // 16))       # pages of a workgroup's step
    assert -(-pages // step) * batch * hkv > 2048
    n_pages = 150
    ends = [0, 1, step - 1, step, step + 1, 2 * step, 2 * step + 1, 3 * step, 8 * step - 1, 8 * step, 8 * step + 1, 9 * step, pages - 1, pages]
    n = rng.choice([min(x, pages) for x in ends], (batch, hkv))
    lengths = np.maximum(n * P - rng.integers(0, P, (batch, hkv)), 0).astype(np.int32)
    table = rng.integers(0, n_pages, (batch, hkv, pages)).astype(np.int32)
    table[rng.random(table.shape) < 0.05] = -1
    table[rng.random(table.shape) < 0.01] = n_pages
    bounds = np.sort(O.as_dtype(rng.standard_normal((n_pages, 2, D)), dtype), axis=1)
    Q = O.as_dtype(rng.standard_normal((batch, hkv * G, D)), dtype)
    p = B.make_paged_params(dtype, "rows", batch, hkv * G, hkv, D, P, pages, n_pages)
    cache = B.PagedCache(None, None, T.i32(table), T.i32(lengths), T.to_device(bounds, dtype))
    q = Q.reshape(batch, hkv, G, D)
    scores = (np.maximum(q, 0).sum(2) @ bounds[:, 1].T + np.minimum(q, 0).sum(2) @ bounds[:, 0].T).astype(np.float32)      # [batch, Hkv, pages of the pool]
    scores = np.concatenate([scores, np.full((batch, hkv, 1), -np.inf, np.float32)], 2)
    for keep, first, last in ((20, 1, 1), (500, 0, 3)):
        (sel,), (got_n,) = B.mixkv_paged_select(p, [cache], [T.to_device(Q, dtype)], keep, first, last)
        sel, got_n = sel.cpu().numpy(), got_n.cpu().numpy()
        for b, h in np.ndindex(batch, hkv):
            row = table[b, h, :-(-int(lengths[b, h]) // P)]
            want = O.select(scores[b, h][np.where((row >= 0) & (row < n_pages), row, n_pages)], keep, first, last)
            assert got_n[b, h] == len(want) and sel[b, h].tolist() == want + [-1] * (keep - len(want)), (b, h, len(row))


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,max_rows", [(64, None), (128, 400)])
def test_logits_of_nearly_two_to_the_25(fmt, dtype, D, max_rows):
    """The largest that the operator is for: fp32 leaves steps of 2 between such logits, so an output is a mean of a few values, and no more than that is
    asked of it here: it is finite, and no larger than they are."""
    rng = np.random.default_rng([48, D])
    lay = T.Layer(rng, fmt, dtype, D, 32, [[620, 500]], 20, fill=True)
    Q = _queries(rng, lay, 6)
    most = max(float(np.abs(Q[0, 3 * h:3 * h + 3] @ O.head(*lay.args(), lay.table, lay.lengths, 0, h)[0].T).max()) for h in range(2))
    for q, scale in ((Q, 0.97 * 2.0 ** 25 / most), (Q * 2.0 ** 25, 0.97 / most)):
        got = T.values(B.mixkv_paged_attention(lay.params(6, scale), [lay.device()], [T.to_device(q, dtype)], max_rows=max_rows)[0])
        for h in range(2):
            v = np.abs(O.head(*lay.args(), lay.table, lay.lengths, 0, h)[1]).max()
            x = got[0, 3 * h:3 * h + 3]
            assert np.isfinite(x).all() and (np.abs(x) <= v * (1 + 2.0 ** -7)).all() and (np.abs(x).max(1) > 0).all()

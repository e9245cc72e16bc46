"""mixkv_paged_append and mixkv_paged_read against the float64 oracle.

Everything is compared bit for bit, whole pools with the rows and pages that nothing may touch: a rotated element is one rounding of a
difference of two products that 64 bits hold exactly (24 by 24 bits), whatever the order, and step, base and codes are decided in
64 bits on either side."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2510_20707_amd import binding as B
from paper_2510_20707_amd import synth
from tests import harness as H
from tests import paged as T

pytestmark = pytest.mark.gpu
KINDS = [("rows", "f32"), ("rows", "bf16"), ("4bit", "bf16")]


def _tables(rng, n, half):
    angle = rng.random((n, half)) * 6.3
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def _append_and_check(rng, lay, hq, K, V, start, count, Q=None, rope=None, max_count=None, strided=None, spoil=None):
    """K, V [n_rows, Hkv, D] float64; strided: the device tensors for them instead of contiguous ones."""
    dt = lay.dtype
    cache = lay.device()
    if spoil:
        spoil(lay, cache)
    Kd, Vd = strided if strided else (T.to_device(K, dt), T.to_device(V, dt))
    Qd = None if Q is None else T.to_device(Q, dt)
    Qo = None if Q is None else torch.full(Q.shape, 7.0, dtype=Qd.dtype, device=T.DEV)
    r = None if rope is None else B.Rope(torch.from_numpy(rope[0]).to(T.DEV), torch.from_numpy(rope[1]).to(T.DEV), T.i32(rope[2]), rope[3])
    rows = B.PagedRows(Kd, Vd, T.i32(start), T.i32(count), Qd, Qo)
    p = lay.params(hq)
    want_q = None if Q is None else np.full(Q.shape, 7.0)
    O.append(*lay.args(), lay.bounds, lay.table, lay.lengths, K, V, np.asarray(start), np.asarray(count), Q, want_q, rope)
    for turn in range(2):                                           # the second call stores the same again
        B.mixkv_paged_append(p, [cache], [rows], r, max_count)
        torch.cuda.synchronize()
        for name, want, got in (("K", lay.K, cache.K_pages), ("V", lay.V, cache.V_pages)):
            bad = np.argwhere(got.cpu().numpy() != want)
            assert len(bad) == 0, f"{name} pages differ in {len(bad)} bytes, the first at {bad[0]} (call {turn})"
        if lay.bounds is not None:
            assert np.array_equal(T.values(cache.K_bounds), lay.bounds)
        if Q is not None:
            assert np.array_equal(T.values(Qo), want_q)
    return cache


def _tokens(rng, lay, hq, counts, pad=0):
    """Packed tokens of a batch, every head of a sequence the same number."""
    batch, hkv = lay.lengths.shape
    starts = np.repeat(np.concatenate([[0], np.cumsum(counts)[:-1]])[:, None], hkv, 1)
    n = int(np.sum(counts)) + pad
    mk = lambda h: O.as_dtype(rng.standard_normal((n, h, lay.D)) * 2 + 0.5, lay.dtype)  # noqa: E731
    return starts, np.repeat(np.asarray(counts)[:, None], hkv, 1), mk(hkv), mk(hkv), mk(hq)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P", [(128, 32), (64, 64), (128, 128), (64, 32)])
def test_one_token_per_sequence(fmt, dtype, D, P):
    # the first row of all, the last of a page, the first of the next, the middle of a tile; a padded sequence
    lens = [1, P, P + 1, 2 * P - 11, 0, 17]
    print(f"[case] append step {fmt} {dtype} D={D} P={P}", flush=True)
    rng = np.random.default_rng([1, D, P])
    lay = T.Layer(rng, fmt, dtype, D, P, np.repeat(np.array(lens)[:, None], 2, 1), 3, bounds=True)
    counts = [min(x, 1) for x in lens]
    start, count, K, V, Q = _tokens(rng, lay, 6, counts)
    n = K.shape[0]
    rope = (*_tables(rng, 300, D // 2), rng.integers(0, 300, (1, n)).astype(np.int32), None)
    _append_and_check(rng, lay, 6, K, V, start, count, Q, rope, max_count=1)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P", [(128, 64), (64, 128), (64, 32)])
def test_ragged_prompts_in_a_padded_batch(fmt, dtype, D, P):
    # prompts that begin inside a page, inside a strip, at a page's beginning; positions beyond the tables; three axes that end inside a
    # group of four pairs, one without any pair; queries of the padding rows stay as they were
    lens, counts = [5 * P // 2, 3 * P, 40, 9, 33], [3 * P // 2 + 7, 3 * P, 3, 0, 21]
    print(f"[case] append prompts {fmt} {dtype} D={D} P={P}", flush=True)
    rng = np.random.default_rng([2, D, P])
    lay = T.Layer(rng, fmt, dtype, D, P, np.repeat(np.array(lens)[:, None], 3, 1), 4, bounds=True)
    start, count, K, V, Q = _tokens(rng, lay, 12, counts, pad=13)
    for sections in (None, (D // 8, 3 * D // 16, 3 * D // 16), (5, 0, D // 2 - 5)):
        axes = 1 if sections is None else 3
        rope = (*_tables(rng, 70, D // 2), rng.integers(-4, 80, (axes, K.shape[0])).astype(np.int32), sections)
        _append_and_check(rng, lay, 12, K, V, start, count, Q, rope, max_count=None if axes == 1 else 2)


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_strided_rows_of_one_projection(fmt, dtype):
    D, P, hq, hkv = 128, 32, 4, 2
    rng = np.random.default_rng(3)
    lay = T.Layer(rng, fmt, dtype, D, P, [[50, 50], [7, 7]], 2)
    start, count, K, V, Q = _tokens(rng, lay, hq, [30, 7])
    x = np.concatenate([Q, K, V], 1)
    xd = T.to_device(x, dtype)
    cache = lay.device()
    out = torch.zeros((x.shape[0], hq, D), dtype=xd.dtype, device=T.DEV)
    rows = B.PagedRows(xd[:, hq:hq + hkv], xd[:, hq + hkv:], T.i32(start), T.i32(count), xd[:, :hq], out)
    B.mixkv_paged_append(lay.params(hq), [cache], [rows])
    O.append(*lay.args(), None, lay.table, lay.lengths, K, V, start, count)
    torch.cuda.synchronize()
    assert np.array_equal(cache.K_pages.cpu().numpy(), lay.K) and np.array_equal(cache.V_pages.cpu().numpy(), lay.V)
    assert np.array_equal(T.values(out), Q)                         # no rotation: copies


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_heads_of_unequal_length_from_one_block(fmt, dtype, D):
    # rows of a packed cache: heads with counts of their own among one another (head stride 0), some of them empty
    P = 32
    rng = np.random.default_rng([4, D])
    lens = np.array([[70, 0, 33], [1, 64, 100]])
    lay = T.Layer(rng, fmt, dtype, D, P, lens, 4, bounds=True)
    start = (np.cumsum(lens.ravel()) - lens.ravel()).reshape(lens.shape)
    rows = O.as_dtype(rng.standard_normal((int(lens.sum()), 1, D)), dtype), O.as_dtype(rng.standard_normal((int(lens.sum()), 1, D)), dtype)
    dev = [T.to_device(x, dtype).expand(-1, 3, -1) for x in rows]
    K, V = (np.repeat(x, 3, 1) for x in rows)
    _append_and_check(rng, lay, 3, K, V, start, lens, strided=dev, max_count=100)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,hkv", [(128, 1), (128, 2), (64, 2)])
@pytest.mark.parametrize("equal", [True, False])
def test_many_query_heads(fmt, dtype, D, hkv, equal):
    # more query heads than a wave takes at once; KV heads with the same rows, or each with its own and their queries alone
    P, hq = 32, 74
    print(f"[case] append queries {fmt} {dtype} D={D} Hkv={hkv} equal={equal}", flush=True)
    rng = np.random.default_rng([30, D, hkv])
    lens = np.array([[70] * hkv, [41] * hkv])
    count = np.array([[37] * hkv, [9] * hkv])
    start = np.array([[0] * hkv, [37] * hkv])
    if not equal:
        count[:, -1] -= 8
        start[:, -1] += 3
    lay = T.Layer(rng, fmt, dtype, D, P, lens, 3, bounds=True)
    K, V, Q = (O.as_dtype(rng.standard_normal((50, h, D)) * 2, dtype) for h in (hkv, hkv, hq))
    rope = (*_tables(rng, 90, D // 2), rng.integers(0, 90, (3, 50)).astype(np.int32), (D // 8, 3 * D // 16, 3 * D // 16))
    _append_and_check(rng, lay, hq, K, V, start, count, Q, rope)
    _append_and_check(rng, lay, hq, K, V, start, count, Q, rope, max_count=2)


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_rows_and_pages_that_do_not_exist_are_left_out(fmt, dtype):
    # dense rows before the first and behind the last, more rows than the head is long, lengths beyond the table, table entries that are
    # no pages of the pool
    D, P = 64, 32
    rng = np.random.default_rng(5)
    lay = T.Layer(rng, fmt, dtype, D, P, [[90, 20], [128 + 40, 60]], 4, bounds=True)
    lay.table[0, 0, 1] = lay.n_pages
    lay.table[1, 1, 0] = -(2 ** 31)
    lay.table[1, 0, 2] = 2 ** 31 - 1
    K, V, Q = (O.as_dtype(rng.standard_normal((50, h, D)), dtype) for h in (2, 2, 2))
    start, count = np.array([[-10, 30], [-2 ** 31, 45]]), np.array([[40, 25], [20, 2 ** 31 - 1]])
    _append_and_check(rng, lay, 2, K, V, start, count, Q, max_count=50)
    _append_and_check(rng, lay, 2, K, V, np.array([[0, 49], [10, 2 ** 31 - 1]]), np.array([[50, 50], [50, -3]]), Q, max_count=1)


def test_values_at_the_ends_of_the_4_bit_format():
    # equal elements (no step), zeros, tiny and huge elements, an offset far above the spread, ties between codes, one outlier
    D, P = 128, 32
    rng = np.random.default_rng(6)
    rows = [np.full(D, 3.0), np.zeros(D), rng.standard_normal(D) * 1e-6, rng.standard_normal(D) * 1e-30, rng.standard_normal(D) * 1e6,
            rng.standard_normal(D) * 3e38, 500 + rng.standard_normal(D), np.tile(np.arange(32) * 0.5, 4), np.where(np.arange(D) == 40, 900.0, 0.01),
            np.tile([-16384.0, 16384.0], D // 2), np.tile(np.arange(16), D // 16) + 0.5, np.where(np.arange(D) % 2, np.inf, -np.inf),
            np.tile(np.arange(32) / 32, 4) * 15]
    x = O.as_dtype(np.array(rows), "bf16")[:, None]
    lay = T.Layer(rng, "4bit", "bf16", D, P, [[len(rows)]], 1)
    _append_and_check(rng, lay, 1, x, x[::-1].copy(), [[0]], [[len(rows)]])


def test_every_code_of_ordinary_rows():
    # 40 000 rows: codes next to a tie are decided as in 64 bits
    D, P, n = 128, 128, 2000
    rng = np.random.default_rng(7)
    lay = T.Layer(rng, "4bit", "bf16", D, P, [[n]], 16)
    K, V = (O.as_dtype(rng.standard_normal((n, 1, D)) * np.exp(rng.standard_normal((n, 1, 1)) * 3) + rng.standard_normal((n, 1, 1)), "bf16") for _ in range(2))
    _append_and_check(rng, lay, 1, K, V, [[0]], [[n]])


def test_codes_of_rows_far_from_zero_and_on_grids():
    # offsets up to 2^12 times the spread, elements on grids of powers of two (exact ties between codes), a few tiny ones among them,
    # groups with elements beyond the format's range
    D, P, n = 128, 128, 2000
    rng = np.random.default_rng(31)
    lay = T.Layer(rng, "4bit", "bf16", D, P, [[n]], 16)
    scale = lambda lo, hi: 2.0 ** rng.integers(lo, hi, (n, 1, 1))  # noqa: E731
    grid = np.round(rng.standard_normal((n, 1, D)) * 16) * scale(-12, 9) + np.round(rng.standard_normal((n, 1, 1)) * 8) * scale(-6, 4)
    K = np.where(rng.random((n, 1, D)) < 0.02, rng.standard_normal((n, 1, D)) * 1e-20, grid)
    V = rng.standard_normal((n, 1, D)) * scale(-14, 13) + rng.standard_normal((n, 1, 1)) * scale(-8, 13)
    K, V = O.as_dtype(K, "bf16"), O.as_dtype(V, "bf16")
    _append_and_check(rng, lay, 1, K, V, [[0]], [[n]])


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P", [(128, 64), (64, 32)])
def test_read_returns_the_newest_rows(fmt, dtype, D, P):
    rng = np.random.default_rng([8, D, P])
    lens = np.array([[3 * P + 5, 40], [0, 2 * P], [1, P + 1]])
    lay = T.Layer(rng, fmt, dtype, D, P, lens, 4, fill=True)
    lay.table[0, 1, 0] = lay.n_pages + 3
    cache, p, n = lay.device(), lay.params(4), 4 * P
    for count, start in ((lens, np.arange(6).reshape(3, 2) * n), (np.array([[7, 33], [5, 200], [1, 2]]), np.arange(6).reshape(3, 2) * n - 3)):
        K, V = np.full((6 * n, 1, D), 7.0), np.full((6 * n, 1, D), -7.0)
        Kd, Vd = T.to_device(K, dtype), T.to_device(V, dtype)
        rows = B.PagedRows(Kd.expand(-1, 2, -1), Vd.expand(-1, 2, -1), T.i32(start), T.i32(count))
        wide = [np.repeat(x, 2, 1) for x in (K, V)]
        O.read(*lay.args(), lay.table, lay.lengths, *wide, start, count)
        B.mixkv_paged_read(p, [cache], [rows], max_count=int(count.max()) if count is lens else 1)
        torch.cuda.synchronize()
        for got, want, fill in ((Kd, wide[0], 7.0), (Vd, wide[1], -7.0)):
            want = np.where(want[:, 0] != fill, want[:, 0], want[:, 1])            # the heads write different rows of one block
            assert np.array_equal(T.values(got)[:, 0], want)


@pytest.mark.parametrize("fmt", ["rows", "4bit"])
def test_more_layers_than_one_launch_takes(fmt):
    D, P, L = 64, 32, 19
    rng = np.random.default_rng(9)
    lays = [T.Layer(rng, fmt, "bf16", D, P, [[10 + l, 10 + l]], 2) for l in range(L)]
    for l in lays:
        l.n_pages = 4
        l.K, l.V = l.K[:4], l.V[:4]
        l.table %= 4
        l.table[0, 1, :] = l.table[0, 0, :] ^ 1
    count = [np.full((1, 2), 10 + l) for l in range(L)]
    data = [[O.as_dtype(rng.standard_normal((40, 2, D)), "bf16") for _ in range(2)] for _ in range(L)]
    caches = [l.device() for l in lays]
    rows = [B.PagedRows(T.to_device(k, "bf16"), T.to_device(v, "bf16"), T.i32(np.zeros((1, 2))), T.i32(n)) for (k, v), n in zip(data, count)]
    B.mixkv_paged_append(lays[0].params(2), caches, rows, max_count=30)
    back = [B.PagedRows(torch.zeros_like(r.K), torch.zeros_like(r.V), r.row_start, r.row_count) for r in rows]
    B.mixkv_paged_read(lays[0].params(2), caches, back, max_count=30)
    torch.cuda.synchronize()
    for l, lay in enumerate(lays):
        O.append(*lay.args(), None, lay.table, lay.lengths, *data[l], np.zeros((1, 2), int), count[l])
        assert np.array_equal(caches[l].K_pages.cpu().numpy(), lay.K) and np.array_equal(caches[l].V_pages.cpu().numpy(), lay.V), l
        K, V = np.zeros((40, 2, D)), np.zeros((40, 2, D))
        O.read(*lay.args(), lay.table, lay.lengths, K, V, np.zeros((1, 2), int), count[l])
        assert np.array_equal(T.values(back[l].K), K) and np.array_equal(T.values(back[l].V), V), l


@pytest.mark.parametrize("mode", ["fixed", "adaptive"])
def test_a_compacted_cache_goes_into_pages(mode):
    wl = synth.WORKLOADS["c2"].with_(name="paged", seq_len=700, text_suffix_start=640, batch=2, budget=96, budget_mode=mode,
                                     budget_floor=16 if mode == "adaptive" else 0, sigma=(0.1, 0.8))
    p, (out,) = H.run_compress(wl, [synth.make_layer(wl, 0)])
    lens, D = out.counts.cpu().numpy(), wl.head_dim
    rng = np.random.default_rng(10)
    lay = T.Layer(rng, "rows", "bf16", D, 64, lens, 8)
    cache, rows = lay.device(), B.compacted_rows(p, out)
    B.mixkv_paged_append(lay.params(wl.n_q_heads), [cache], [rows])
    torch.cuda.synchronize()
    off = np.arange(wl.n_kv_heads + 1)[None].repeat(2, 0) * wl.budget if mode == "fixed" else out.offsets.cpu().numpy()
    for b, h in np.ndindex(*lens.shape):
        k, v = O.head(*lay.args()[:4], cache.K_pages.cpu().numpy(), cache.V_pages.cpu().numpy(), lay.table, lens, b, h)
        at = slice(off[b, h], off[b, h] + lens[b, h])
        assert np.array_equal(k, T.values(out.K_out[b].reshape(-1, D)[at])) and np.array_equal(v, T.values(out.V_out[b].reshape(-1, D)[at]))

"""mixkv_paged_evict against the oracle: what is kept and moved is compared exactly."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2510_20707_amd import binding as B
from tests import paged as T

pytestmark = pytest.mark.gpu
KINDS = [("rows", "f32"), ("rows", "bf16"), ("4bit", "bf16")]


def _into(rng, lay, rows, none=()):
    """A table of free pages for `rows` rows of each head, and pages enough in the layer's pools."""
    units, width = lay.lengths.size, lay.table.shape[2]
    used = set(lay.table.reshape(-1).tolist())
    need = -(-np.maximum(np.asarray(rows).reshape(-1), 0) // lay.P)
    free = [i for i in rng.permutation(lay.n_pages).tolist() if i not in used]
    table, at = np.full((units, width), -1, np.int32), 0
    for u in range(units):
        k = min(int(need[u]), width)
        table[u, :k] = free[at:at + k]
        at += k
    for u, i in none:
        table[u, i] = [-1, lay.n_pages, 2 ** 31 - 1][i % 3]
    return table.reshape(lay.table.shape)


def _check(rng, lay, weights, keep, max_keep, first=0, last=0, none=(), own_pool=True, max_rows=None):
    into = _into(rng, lay, np.minimum(keep, max_keep), none)
    cache, w = lay.device(), torch.from_numpy(weights).to(T.DEV)
    other = lay.device()
    w_into = w if own_pool else torch.full_like(w, 5.0)
    pools = cache if own_pool else other
    target = B.PagedCache(pools.K_pages, pools.V_pages, T.i32(into), T.i32(np.full(lay.lengths.shape, 99)), pools.K_bounds)
    (kept,) = B.mixkv_paged_evict(lay.params(lay.lengths.shape[1]), [cache], [target], [w], [T.i32(keep)], max_keep, first, last, weights_into=[w_into], max_rows=max_rows)
    K, V = lay.K.copy(), lay.V.copy()
    bounds = None if lay.bounds is None else lay.bounds.copy()
    want_w = weights.copy() if own_pool else np.full_like(weights, 5.0)
    src = (lay.fmt, lay.dtype, lay.P, lay.D, lay.K, lay.V)
    want, n = O.evict(src, lay.table, lay.lengths, into, weights, want_w, keep, max_keep, first, last, K, V, bounds)
    assert np.array_equal(target.lengths.cpu().numpy(), n)
    assert np.array_equal(kept.cpu().numpy(), want)
    assert np.array_equal(target.K_pages.cpu().view(torch.uint8).numpy().reshape(K.shape), K) and np.array_equal(target.V_pages.cpu().view(torch.uint8).numpy().reshape(V.shape), V)
    assert np.array_equal(w_into.cpu().numpy(), want_w, equal_nan=True)
    if bounds is not None:
        assert np.array_equal(T.values(target.K_bounds), bounds)
    if not own_pool:                                   # the caches' own pages and weights are not touched
        assert np.array_equal(cache.K_pages.cpu().view(torch.uint8).numpy().reshape(K.shape), lay.K) and np.array_equal(w.cpu().numpy(), weights, equal_nan=True)
    return want, n


def _weights(rng, lay, zeros=0.2):
    return (np.exp(2 * rng.standard_normal((lay.n_pages, lay.P))) * (rng.random((lay.n_pages, lay.P)) >= zeros)).astype(np.float32)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("D,P", [(128, 64), (64, 32), (128, 32), (64, 128), (128, 128)])
@pytest.mark.parametrize("own_pool", [True, False])
def test_heads_of_unequal_length_and_budget(fmt, dtype, D, P, own_pool):
    print(f"[case] evict {fmt} {dtype} D={D} P={P}", flush=True)
    rng = np.random.default_rng([81, D, P])
    lens = np.array([[300, 1, 31], [32, 33, P], [P + 1, 2 * P - 1, 0], [127, 128, 129], [257, 96, 160]])
    keep = np.array([[100, 1, 40], [31, 32, 1], [P, P + 1, 5], [0, -3, 129], [256, 33, 500]], np.int32)
    lay = T.Layer(rng, fmt, dtype, D, P, lens, 10, spare=60, bounds=True, fill=True)
    w = _weights(rng, lay)
    for first, last, most in ((0, 0, 300), (4, 16, 300), (40, 300, 130), (2 ** 31 - 1, 0, 300), (0, 2 ** 31 - 1, 64)):
        _check(rng, lay, w, keep, most, first, last, own_pool=own_pool)


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_pages_that_are_none(fmt, dtype):
    rng = np.random.default_rng(82)
    lay = T.Layer(rng, fmt, dtype, 64, 32, [[200, 150], [1000, -5]], 8, spare=30, bounds=True, fill=True)
    w = _weights(rng, lay)
    lay.table[0, 0, 1], lay.table[0, 1, 0], lay.table[0, 1, 4] = lay.n_pages, -7, 2 ** 31 - 1
    lay.table[1, 0, 3:] = -1
    for keep in (np.full((2, 2), 90, np.int32), np.full((2, 2), 256, np.int32)):
        want, n = _check(rng, lay, w, keep, 256, 3, 10, none=[(0, 1), (1, 2), (2, 0)])
    assert n.tolist() == [[168, 96], [96, 0]]


@pytest.mark.parametrize("what", ["equal", "zeros of both signs", "two values", "infinite and NaN", "negative", "neighbours"])
@pytest.mark.parametrize("n", [90, 1500, 20000])
def test_weights_that_are_equal_or_no_numbers(what, n):
    rng = np.random.default_rng([83, n])
    D, P = 64, 128
    lay = T.Layer(rng, "rows", "bf16", D, P, [[n, n - 7]], -(-n // P), spare=2 * (-(-n // P)) + 2)
    shape = (lay.n_pages, P)
    w = {"equal": np.full(shape, 2.0), "zeros of both signs": np.where(rng.random(shape) < 0.5, 0.0, -0.0), "two values": rng.integers(0, 2, shape) + 1.0,
         "infinite and NaN": rng.choice([np.inf, -np.inf, np.nan, -np.nan, 1.0, 3.0], shape), "negative": -rng.integers(1, 5, shape).astype(float),
         "neighbours": 1.0 + rng.integers(0, 4, shape) * 2.0 ** -23}[what].astype(np.float32)
    lay.fmt = "rows"
    for keep, first, last in ((n // 3, 0, 0), (n // 2, 4, 20), (1, 0, 0), (n - 1, 1, 1)):
        cache = lay.device()
        into = B.PagedCache(cache.K_pages, cache.V_pages, T.i32(_into(rng, lay, np.full((1, 2), keep))), T.i32(np.zeros((1, 2))))
        (kept,) = B.mixkv_paged_evict(lay.params(2), [cache], [into], [torch.from_numpy(w).to(T.DEV)], [T.i32(np.full((1, 2), keep))], keep, first, last)
        for h in range(2):
            j = np.arange(n - 7 * h)
            want = O.evicted(w[lay.table[0, h, j // P], j % P].astype(np.float64), np.ones(len(j), bool), keep, first, last)
            assert kept[0, h, :len(want)].tolist() == want and (kept[0, h, len(want):] == -1).all(), (what, keep, h)


@pytest.mark.parametrize("n", [3000, 8193, 16384, 16385, 40000, 70000, 140000, 300000])
def test_long_heads(n):
    """Heads around what a workgroup takes at once, the choice compared with a sort."""
    _long(n, n)


@pytest.mark.parametrize("n,max_rows", [(3000, 100), (6000, 3000), (20000, 16000), (20000, 16385), (40000, 17000)])
def test_heads_longer_than_the_host_said(n, max_rows):
    """They are served all the same, whichever kernel was chosen for shorter ones."""
    _long(n, max_rows)


def _long(n, max_rows):
    print(f"[case] evict long n={n} max_rows={max_rows}", flush=True)
    rng = np.random.default_rng([84, n])
    D, P = 64, 32
    pages = -(-n // P)
    lens = np.array([[n, n // 2, 5]], np.int32)
    n_pages = 2 * pages + 10
    table = np.full((1, 3, pages), -1, np.int32)
    ids = rng.permutation(n_pages)
    table[0, 0] = ids[:pages]
    table[0, 1, :-(-(n // 2) // P)] = ids[pages:pages - (-(n // 2) // P)]
    table[0, 2, 0] = ids[-1]
    w = np.exp(3 * rng.standard_normal((n_pages, P))).astype(np.float32)
    w[rng.random(w.shape) < 0.5] = 0.0
    K = torch.randn((n_pages, P, D), device=T.DEV).bfloat16()
    V = torch.randn((n_pages, P, D), device=T.DEV).bfloat16()
    p = B.make_paged_params("bf16", "rows", 1, 3, 3, D, P, pages, n_pages)
    cache = B.PagedCache(K, V, T.i32(table), T.i32(lens))
    for share, first, last in ((0.1, 4, 64), (0.7, 0, 0), (0.97, 100, 1000)):
        keep = np.maximum((lens * share).astype(np.int32), 1)
        out = [torch.zeros_like(K), torch.zeros_like(V)]
        into_table = np.full((1, 3, pages), -1, np.int32)
        at = 0
        for h in range(3):
            m = -(-int(keep[0, h]) // P)
            into_table[0, h, :m] = np.arange(at, at + m)
            at += m
        into = B.PagedCache(*out, T.i32(into_table), T.i32(np.zeros((1, 3))))
        w_into = torch.zeros((n_pages, P), device=T.DEV)
        (kept,) = B.mixkv_paged_evict(p, [cache], [into], [torch.from_numpy(w).to(T.DEV)], [T.i32(keep)], int(keep.max()), first, last, weights_into=[w_into], max_rows=max_rows)
        kept = kept.cpu().numpy()
        assert np.array_equal(into.lengths.cpu().numpy(), keep)
        for h in range(3):
            j = np.arange(lens[0, h])
            x = w[table[0, h, j // P], j % P].astype(np.float64)
            x[j < first] = np.inf
            x[j >= lens[0, h] - last] = np.inf
            best = np.sort(np.argsort(-x, kind="stable")[:keep[0, h]])
            assert np.array_equal(kept[0, h, :keep[0, h]], best) and (kept[0, h, keep[0, h]:] == -1).all(), (h, share)
            src = torch.from_numpy(table[0, h, best // P].astype(np.int64)).to(T.DEV)
            i = torch.arange(len(best), device=T.DEV)
            dst = torch.from_numpy(into_table[0, h]).to(T.DEV).long()[i // P]
            r = torch.from_numpy(best % P).to(T.DEV)
            assert torch.equal(out[0][dst, i % P], K[src, r]) and torch.equal(out[1][dst, i % P], V[src, r])
            assert np.array_equal(w_into.cpu().numpy()[into_table[0, h, np.arange(len(best)) // P], np.arange(len(best)) % P], w[table[0, h, best // P], best % P])


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_long_heads_with_missing_pages_beside_short_ones(fmt, dtype):
    rng = np.random.default_rng(86)
    lay = T.Layer(rng, fmt, dtype, 64, 128, [[18000, 0], [40, 16700]], 141, spare=220, bounds=True, fill=False)
    lay.K &= np.uint8(0xbf)                            # numbers below 2, of both signs, and steps and bases of the same kind
    lay.table[0, 0, 3], lay.table[0, 0, 100], lay.table[1, 1, 0] = -1, lay.n_pages, -9
    w = _weights(rng, lay)
    for keep, first, last in (([[9000, 5], [40, 16000]], 10, 300), ([[17999, 1], [7, 0]], 0, 0)):
        _check(rng, lay, w, np.array(keep, np.int32), 17999, first, last, own_pool=False)


def test_long_heads_of_several_layers():
    """Each layer's choice is what a call for it alone gives."""
    rng = np.random.default_rng(87)
    n, P, D = 17500, 128, 64
    pages = -(-n // P)
    p = B.make_paged_params("bf16", "rows", 2, 2, 2, D, P, pages, 8 * pages)
    caches, into, ws, keeps = [], [], [], []
    for i in range(3):
        ids = rng.permutation(8 * pages).astype(np.int32)
        K, V = (torch.randn((8 * pages, P, D), device=T.DEV).bfloat16() for _ in range(2))
        caches.append(B.PagedCache(K, V, T.i32(ids[:4 * pages].reshape(2, 2, pages)), T.i32([[n, n - 1000 * i], [30, 16385 + i]])))
        into.append(lambda K=K, V=V, ids=ids: B.PagedCache(K.clone(), V.clone(), T.i32(ids[4 * pages:].reshape(2, 2, pages)), T.i32(np.zeros((2, 2)))))
        ws.append(torch.from_numpy(np.exp(rng.standard_normal((8 * pages, P))).astype(np.float32)).to(T.DEV))
        keeps.append(T.i32([[8000, 9000], [20, 16000]]))
    together = [z() for z in into]
    kept = B.mixkv_paged_evict(p, caches, together, ws, keeps, 16000, 4, 64)
    for i in range(3):
        alone = into[i]()
        (one,) = B.mixkv_paged_evict(p, [caches[i]], [alone], [ws[i]], [keeps[i]], 16000, 4, 64)
        assert torch.equal(one, kept[i]) and torch.equal(alone.lengths, together[i].lengths)
        assert torch.equal(alone.K_pages, together[i].K_pages) and torch.equal(alone.V_pages, together[i].V_pages)


def test_many_layers_and_a_captured_call():
    """More layers than a launch takes; captured on a side stream and replayed with other weights."""
    rng = np.random.default_rng(85)
    layers = [T.Layer(rng, "rows", "f32", 64, 32, [[150 + i, 90]], 7, spare=9, fill=True) for i in range(27)]
    n_pages = max(l.n_pages for l in layers)
    caches, into, ws, keeps, kepts = [], [], [], [], []
    for lay in layers:
        c = lay.device()
        grow = lambda t: torch.cat((t, t[:1].expand(n_pages - t.shape[0], *t.shape[1:]))).contiguous()  # noqa: E731
        caches.append(B.PagedCache(grow(c.K_pages.view(lay.n_pages, -1)), grow(c.V_pages.view(lay.n_pages, -1)), c.page_table, c.lengths))
        into.append(B.PagedCache(caches[-1].K_pages, caches[-1].V_pages, T.i32(_into(rng, lay, [60, 50])), T.i32(np.zeros((1, 2)))))
        ws.append(torch.zeros((n_pages, 32), device=T.DEV))
        keeps.append(T.i32([[60, 50]]))
        kepts.append(torch.zeros((1, 2, 60), dtype=torch.int32, device=T.DEV))
    p = layers[0].params(2)
    p.n_pages = n_pages
    call = B.PreparedPagedEvict(p, caches, into, ws, keeps, kepts, 4, 8, weights_into=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call.run(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call.run()
    for turn in range(3):
        host = [np.exp(rng.standard_normal((n_pages, 32))).astype(np.float32) for _ in layers]
        for w, x in zip(ws, host):
            w.copy_(torch.from_numpy(x))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for lay, x, kept, z in zip(layers, host, kepts, into):
            for h, keep in enumerate((60, 50)):
                j = np.arange(lay.lengths[0, h])
                want = O.evicted(x[lay.table[0, h, j // 32], j % 32].astype(np.float64), np.ones(len(j), bool), keep, 4, 8)
                assert kept[0, h, :keep].tolist() == want
            assert z.lengths.tolist() == [[60, 50]]

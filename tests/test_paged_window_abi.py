"""Host-side checks of mixkv_paged_window_attention, mixkv_paged_weights and mixkv_paged_evict that need no GPU: struct layouts, sizes, and every
refusal, which comes before anything is launched (the addresses here are never dereferenced)."""
import ctypes as C
import weakref

import pytest
import torch

from paper_2510_20707_amd import binding as B
from tests.test_paged_abi import _caches, _params

INVALID, UNSUPPORTED, SMALL = B.MIXKV_ERR_INVALID_ARG, B.MIXKV_ERR_UNSUPPORTED, B.MIXKV_ERR_WORKSPACE_TOO_SMALL


def _queries(n=1, **kw):
    arr = (B.MixkvPagedQueries * n)()
    for i in range(n):
        f = dict(Q=0x10000000, q_stride_n=28 * 128, q_stride_h=128, row_start=0x60000, row_count=0x70000, out=0x20000000, lse=0x30000000)
        f.update(kw)
        arr[i] = B.MixkvPagedQueries(*f.values())
    return arr


def _attend(p=None, caches=None, queries=None, n=1, rows=100, window=10, first=2, count=5, most=1000, ws=0x900000, size=1 << 40):
    return B.lib().mixkv_paged_window_attention(C.byref(p or _params()), caches or _caches(max(n, 1)), queries or _queries(max(n, 1)), n, rows, window, first, count,
                                                most, ws, size, None)


def _weigh(p=None, caches=None, queries=None, n=1, rows=100, window=10, first=2, count=5, most=1000, ws=0x900000, size=1 << 40, weights=0x40000000):
    w = (C.c_void_p * max(n, 1))(*[weights] * max(n, 1)) if weights is not None else None
    return B.lib().mixkv_paged_weights(C.byref(p or _params()), caches or _caches(max(n, 1)), queries or _queries(max(n, 1)), w, n, rows, window, first, count, most,
                                       ws, size, None)


def _evict(p=None, caches=None, into=None, n=1, keep=100, first=4, last=8, rows=1000, ws=0x900000, size=1 << 40, null=False, **kw):
    arr = (B.MixkvPagedEvictLayer * max(n, 1))()
    for i in range(max(n, 1)):
        arr[i] = B.MixkvPagedEvictLayer(*{**dict(weights=0x1000, weights_into=0x1000, keep=0x2000, kept=0x3000, n_kept=0x4000), **kw}.values())
    return B.lib().mixkv_paged_evict(C.byref(p or _params()), caches or _caches(max(n, 1)), into or _caches(max(n, 1), page_table=0x80000), None if null else arr, n, keep,
                                     first, last, rows, ws, size, None)


def test_struct_layouts():
    assert C.sizeof(B.MixkvPagedQueries) == 7 * 8 and C.sizeof(B.MixkvPagedEvictLayer) == 5 * 8


@pytest.mark.parametrize("kw,status", [(dict(head_dim=96), UNSUPPORTED), (dict(page_rows=16), UNSUPPORTED), (dict(dtype="f32"), UNSUPPORTED), (dict(batch=0), INVALID),
                                       (dict(max_pages=1 << 25), UNSUPPORTED), (dict(softmax_scale=float("nan")), INVALID)])
def test_bad_params(kw, status):
    p, n = _params(**kw), C.c_size_t()
    assert _attend(p) == _weigh(p) == _evict(p) == status
    assert B.lib().mixkv_paged_window_attention_workspace_size(C.byref(p), 1, 10, 5, 0, 1, 100, C.byref(n)) == status
    assert B.lib().mixkv_paged_weights_workspace_size(C.byref(p), 1, 10, 5, 0, 1, 100, C.byref(n)) == status
    assert B.lib().mixkv_paged_evict_workspace_size(C.byref(p), 1, 100, C.byref(n)) == status


@pytest.mark.parametrize("kw", [dict(rows=0), dict(rows=-1), dict(window=0), dict(window=-5), dict(first=-1), dict(count=0), dict(most=0), dict(n=0), dict(n=129)])
def test_bad_sizes(kw):
    assert _attend(**kw) == _weigh(**kw) == INVALID


def test_too_many_rows():
    assert _attend(rows=2 ** 31 // 28 + 1) == _weigh(rows=2 ** 31 // 28 + 1) == UNSUPPORTED


@pytest.mark.parametrize("kw,both", [(dict(Q=0), True), (dict(Q=0x10000008), True), (dict(q_stride_n=100), True), (dict(q_stride_h=3), True), (dict(q_stride_h=-128), True),
                                     (dict(row_start=0), True), (dict(row_count=0x70002), True), (dict(lse=0x30000002), True), (dict(out=0), False), (dict(out=0x20000004), False),
                                     (dict(out=0x10000000), False), (dict(out=0x10000000 + 99 * 28 * 256), False), (dict(lse=0x10000100), False), (dict(lse=0x20000100), False)])
def test_bad_queries(kw, both):
    assert _attend(queries=_queries(**kw)) == INVALID
    if both:
        assert _weigh(queries=_queries(**kw)) == INVALID


def test_what_only_one_of_them_needs():
    assert _weigh(queries=_queries(lse=0)) == INVALID and _weigh(weights=0) == INVALID and _weigh(weights=None) == INVALID and _weigh(weights=0x40000008) == INVALID
    assert _weigh(caches=_caches(K_pages=0)) == INVALID and _attend(caches=_caches(V_pages=0)) == INVALID


@pytest.mark.parametrize("kw", [dict(K_pages=0x10008), dict(page_table=0), dict(lengths=0), dict(lengths=0x50002)])
def test_bad_caches(kw):
    assert _attend(caches=_caches(**kw)) == _weigh(caches=_caches(**kw)) == _evict(caches=_caches(**kw)) == INVALID


def test_workspaces():
    for count, most in ((1, 8000), (100, 100000)):
        p = _params(max_pages=4000)
        need = B.mixkv_paged_window_attention_workspace_size(p, 1, 100, 1 << 30, 0, count, most)
        assert need > 0 and need % 256 == 0
        kw = dict(p=p, window=1 << 30, first=0, count=count, most=most)
        assert _attend(ws=None, **kw) == _attend(ws=0x900080, **kw) == INVALID and _attend(size=need - 256, **kw) == SMALL
    assert B.mixkv_paged_window_attention_workspace_size(_params(), 1, 100, 64, 0, 1, 1 << 30) == 0        # a short window: whole
    p = _params(dtype="f32", format="rows", max_pages=4000)
    assert B.mixkv_paged_window_attention_workspace_size(p, 1, 16384, 1 << 30, 0, 16384, 16384) == 0        # fp32 prompts: groups enough, no partial sums
    for layers in (1, 32):                                                             # first rows, which every row sees, do not make the sums of all keys longer
        few, more = (B.mixkv_paged_weights_workspace_size(_params(max_pages=2048), layers, 131072, 1024, first, 131072, 131072) for first in (0, 16))
        assert few <= more <= few + layers * 2 * 4 * 256 * 512 * 4
    for size in (B.lib().mixkv_paged_window_attention_workspace_size, B.lib().mixkv_paged_weights_workspace_size):
        assert size(C.byref(_params()), 1, 10, 5, 0, 1, 100, None) == INVALID and size(C.byref(_params()), 0, 10, 5, 0, 1, 100, C.byref(C.c_size_t())) == INVALID
    assert B.lib().mixkv_paged_evict_workspace_size(C.byref(_params()), 1, 0, C.byref(C.c_size_t())) == INVALID


@pytest.mark.parametrize("kw", [dict(keep=0), dict(keep=16 * 64 + 1), dict(first=-1), dict(last=-1), dict(rows=0), dict(n=0), dict(n=129), dict(null=True), dict(weights=0),
                                dict(keep_=0), dict(kept=0), dict(n_kept=0), dict(weights=0x1008), dict(weights_into=0x1001), dict(kept=0x3002), dict(n_kept=0x50000),
                                dict(n_kept=0x2000)])
def test_bad_evictions(kw):
    if "keep_" in kw:
        arr = (B.MixkvPagedEvictLayer * 1)(B.MixkvPagedEvictLayer(0x1000, 0, 0, 0x3000, 0x4000))
        assert B.lib().mixkv_paged_evict(C.byref(_params()), _caches(), _caches(page_table=0x80000), arr, 1, 100, 0, 0, 1000, 0x900000, 1 << 40, None) == INVALID
    else:
        assert _evict(**kw) == INVALID


@pytest.mark.parametrize("kw", [dict(K_pages=0), dict(V_pages=0x10000), dict(K_bounds=0x30004), dict(page_table=0), dict(page_table=0x40000), dict(page_table=0x80002)])
def test_bad_targets(kw):
    assert _evict(into=_caches(**{"page_table": 0x80000, **kw})) == INVALID


# ---- the binding: shapes and types are checked, and what a prepared call was prepared over stays
CPU = torch.device("cpu")


def _parts():
    p = B.make_paged_params("bf16", "rows", 1, 4, 2, 64, 32, 3, 5)
    f = lambda *shape: torch.zeros(shape)  # noqa: E731
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    b = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)  # noqa: E731
    q = B.PagedQueries(b(6, 4, 64), i(1, 2), i(1, 2), b(6, 4, 64), f(6, 4))
    return p, B.alloc_paged_cache(p, CPU), B.alloc_paged_cache(p, CPU), q, f(5, 32), f(5, 32), i(1, 2), i(1, 2, 40)


CALLS = {
    "attention": lambda p, c, into, q, w, w2, keep, kept: B.PreparedPagedWindowAttention(p, [c], [q], 8, 1),
    "weights": lambda p, c, into, q, w, w2, keep, kept: B.PreparedPagedWeights(p, [c], [q], [w], 8, 1),
    "evict": lambda p, c, into, q, w, w2, keep, kept: B.PreparedPagedEvict(p, [c], [into], [w], [keep], [kept], weights_into=[w2]),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_prepared_call_holds_its_tensors(name, monkeypatch):
    monkeypatch.setattr(B, "_paged_device", lambda caches: CPU)
    parts = _parts()
    call = CALLS[name](*parts)
    p, c, into, q, w, w2, keep, kept = parts
    refs = [weakref.ref(t) for t in ([c.K_pages, c.page_table, c.lengths] + ([q.Q, q.row_start, q.row_count, q.lse] if name != "evict" else [into.V_pages, into.lengths, keep, kept, w2])
                                     + ([w] if name != "attention" else [q.out, c.V_pages]))]
    p.batch = 77                                          # the call's own params are what it was prepared with
    assert call.p.batch == 1
    del parts, p, c, into, q, w, w2, keep, kept
    assert all(r() is not None for r in refs)
    del call
    assert all(r() is None for r in refs)


@pytest.mark.parametrize("name,spoil", [
    ("attention", lambda s: setattr(s[3], "Q", s[3].Q[:, :3])), ("attention", lambda s: setattr(s[3], "Q", s[3].Q.float())),
    ("attention", lambda s: setattr(s[3], "Q", s[3].Q.transpose(1, 2).contiguous().transpose(1, 2))), ("attention", lambda s: setattr(s[3], "out", None)),
    ("attention", lambda s: setattr(s[3], "out", s[3].out[:5])), ("attention", lambda s: setattr(s[3], "lse", s[3].lse.half())),
    ("attention", lambda s: setattr(s[3], "row_start", s[3].row_start.long())), ("attention", lambda s: setattr(s[1], "V_pages", None)),
    ("weights", lambda s: setattr(s[3], "lse", None)), ("weights", lambda s: setattr(s[3], "lse", s[3].lse.t().contiguous().t())), ("weights", lambda s: setattr(s[1], "K_pages", None)),
    ("weights", lambda s: s.__setitem__(4, s[4][:4])), ("evict", lambda s: s.__setitem__(4, s[4].t().contiguous().t())), ("evict", lambda s: s.__setitem__(5, s[5].double())),
    ("evict", lambda s: s.__setitem__(6, s[6][0])), ("evict", lambda s: s.__setitem__(7, s[7].long())), ("evict", lambda s: setattr(s[2], "lengths", s[2].lengths[0])),
    ("evict", lambda s: setattr(s[2], "K_pages", s[2].K_pages[:4])),
])
def test_shapes_and_types_are_checked(name, spoil, monkeypatch):
    monkeypatch.setattr(B, "_paged_device", lambda caches: CPU)
    parts = list(_parts())
    spoil(parts)
    with pytest.raises(ValueError):
        CALLS[name](*parts)

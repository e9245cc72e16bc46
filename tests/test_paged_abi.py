"""Host-side checks of the paged cache's entry points that need no GPU: struct layouts, sizes, and every refusal, which comes
before anything is launched (the addresses here are never dereferenced)."""
import ctypes as C

import pytest

from paper_2510_20707_amd import binding as B

INVALID, UNSUPPORTED = B.MIXKV_ERR_INVALID_ARG, B.MIXKV_ERR_UNSUPPORTED


def _params(**kw):
    base = dict(dtype="bf16", format="4bit", batch=2, n_q_heads=28, n_kv_heads=4, head_dim=128, page_rows=64, max_pages=16, n_pages=40)
    base.update(kw)
    return B.make_paged_params(**base)


def _caches(n=1, **kw):
    arr = (B.MixkvPagedCache * n)()
    for i in range(n):
        f = dict(K_pages=0x10000, V_pages=0x20000, K_bounds=0x30000, page_table=0x40000, lengths=0x50000)
        f.update(kw)
        arr[i] = B.MixkvPagedCache(*f.values())
    return arr


def _rows(n=1, **kw):
    arr = (B.MixkvPagedRows * n)()
    for i in range(n):
        f = dict(K=0x100000, V=0x200000, stride_n=128 * 4, stride_h=128, row_start=0x60000, row_count=0x70000, Q=0x300000, q_stride_n=28 * 128,
                 q_stride_h=128, Q_out=0x10000000)
        f.update(kw)
        arr[i] = B.MixkvPagedRows(*f.values())
    return arr


def _rope(**kw):
    f = dict(cos=0x1000, sin=0x2000, n_positions=100, positions=0x3000, n_axes=3, sections=(16, 24, 24))
    f.update(kw)
    return B.MixkvRope(f["cos"], f["sin"], f["n_positions"], f["positions"], f["n_axes"], (C.c_int32 * 3)(*f["sections"]))


def _select(p=None, caches=None, n=1, keep=8, first=1, last=1, ws=0x900000, size=1 << 40, null=False, **kw):
    arr = (B.MixkvPagedSelectLayer * max(n, 1))()
    for i in range(max(n, 1)):
        arr[i] = B.MixkvPagedSelectLayer(*{**dict(Q=0x1000, selected=0x2000, n_selected=0x3000), **kw}.values())
    return B.lib().mixkv_paged_select(C.byref(p or _params()), _caches(max(n, 1)) if caches is None else caches, None if null else arr, n, keep, first, last,
                                      ws, size, None)


def _attend(p=None, caches=None, n=1, most=8, rows=1000, ws=0x900000, size=1 << 40, null=False, second=None, **kw):
    arr = (B.MixkvPagedAttentionLayer * max(n, 1))()
    for i in range(max(n, 1)):
        arr[i] = B.MixkvPagedAttentionLayer(*{**dict(Q=0x1000, out=0x2000, selected=0x3000, n_selected=0x4000), **kw, **(second or {} if i else {})}.values())
    return B.lib().mixkv_paged_attention(C.byref(p or _params()), _caches(max(n, 1)) if caches is None else caches, None if null else arr, n, most, rows, ws,
                                         size, None)


def test_struct_layouts():
    assert C.sizeof(B.MixkvPagedParams) == 10 * 4 and C.sizeof(B.MixkvPagedCache) == 5 * 8 and C.sizeof(B.MixkvPagedRows) == 10 * 8
    assert C.sizeof(B.MixkvRope) == 16 + 8 + 8 + 16
    assert C.sizeof(B.MixkvPagedSelectLayer) == 3 * 8 and C.sizeof(B.MixkvPagedAttentionLayer) == 4 * 8


@pytest.mark.parametrize("kw,size", [(dict(), 64 * 128 * 5 // 8), (dict(head_dim=64, page_rows=32), 32 * 64 * 5 // 8),
                                     (dict(format="rows"), 64 * 128 * 2), (dict(format="rows", dtype="f32", page_rows=128), 128 * 128 * 4)])
def test_page_bytes(kw, size):
    assert B.mixkv_page_bytes(_params(**kw)) == size
    assert B.lib().mixkv_page_bytes(C.byref(_params()), None) == INVALID and B.lib().mixkv_page_bytes(None, C.byref(C.c_size_t())) == INVALID


@pytest.mark.parametrize("kw,status", [(dict(head_dim=96), UNSUPPORTED), (dict(page_rows=16), UNSUPPORTED), (dict(page_rows=48), UNSUPPORTED),
                                       (dict(dtype="f32"), UNSUPPORTED),                       # 4-bit pages of fp32 rows
                                       (dict(batch=0), INVALID), (dict(n_q_heads=30), INVALID), (dict(n_kv_heads=0), INVALID),
                                       (dict(max_pages=0), INVALID), (dict(n_pages=0), INVALID), (dict(max_pages=1 << 25), UNSUPPORTED),
                                       (dict(batch=1 << 14), UNSUPPORTED),
                                       (dict(softmax_scale=0.0), INVALID), (dict(softmax_scale=float("nan")), INVALID),
                                       (dict(softmax_scale=float("inf")), INVALID), (dict(softmax_scale=-1.0), INVALID)])
def test_bad_params_are_rejected_everywhere(kw, status):
    p, L = _params(**kw), B.lib()
    with pytest.raises(B.MixkvError) as e:
        B.mixkv_page_bytes(p)
    assert e.value.status == status
    assert L.mixkv_paged_append(C.byref(p), _caches(), _rows(), 1, None, 10, 1, None) == status
    assert L.mixkv_paged_read(C.byref(p), _caches(), _rows(), 1, 10, 1, None) == status
    assert _select(p=p) == _attend(p=p) == status
    for size in (lambda: B.mixkv_paged_select_workspace_size(p, 1), lambda: B.mixkv_paged_attention_workspace_size(p, 1, 100)):
        with pytest.raises(B.MixkvError) as e:
            size()
        assert e.value.status == status


@pytest.mark.parametrize("field,value", [("dtype", 2), ("format", 2), ("format", -1)])
def test_unknown_enums_are_rejected(field, value):
    p = _params()
    setattr(p, field, value)
    with pytest.raises(B.MixkvError) as e:
        B.mixkv_page_bytes(p)
    assert e.value.status == INVALID


@pytest.mark.parametrize("kw", [dict(K_pages=0), dict(V_pages=0), dict(K_pages=0x10008), dict(V_pages=0x10000), dict(K_bounds=0x30004), dict(page_table=0),
                                dict(lengths=0), dict(lengths=0x50002)])
def test_bad_caches_are_rejected(kw):
    p, L = _params(), B.lib()
    assert L.mixkv_paged_append(C.byref(p), _caches(**kw), _rows(), 1, None, 10, 1, None) == INVALID
    assert L.mixkv_paged_read(C.byref(p), _caches(**kw), _rows(), 1, 10, 1, None) == INVALID


@pytest.mark.parametrize("kw,read", [(dict(K=0), True), (dict(V=0x200008), True), (dict(stride_n=64), True), (dict(stride_h=-128), True), (dict(stride_n=516), True),
                                     (dict(stride_h=4), True), (dict(row_start=0), True), (dict(row_count=0x70001), True), (dict(Q=0), False),
                                     (dict(Q_out=0), False), (dict(Q_out=0x300000), False), (dict(Q_out=0x100400), False), (dict(Q_out=0x1f0000), False),
                                     (dict(Q=0x300008), False), (dict(q_stride_n=100), False), (dict(q_stride_h=3), False)])
def test_bad_rows_are_rejected(kw, read):
    p, L = _params(), B.lib()
    assert L.mixkv_paged_append(C.byref(p), _caches(), _rows(**kw), 1, None, 30, 1, None) == INVALID
    if read:
        assert L.mixkv_paged_read(C.byref(p), _caches(), _rows(**kw), 1, 30, 1, None) == INVALID


def test_queries_come_for_every_layer_or_none():
    rows = _rows(2)
    rows[1] = _rows(Q=0, Q_out=0)[0]
    assert B.lib().mixkv_paged_append(C.byref(_params()), _caches(2), rows, 2, None, 10, 1, None) == INVALID


@pytest.mark.parametrize("kw", [dict(cos=0), dict(sin=0), dict(cos=0x1004), dict(positions=0), dict(n_positions=0), dict(n_axes=2), dict(n_axes=0),
                                dict(sections=(16, 24, 25)), dict(sections=(-1, 40, 25)), dict(sections=(2 ** 31 - 1, 2 ** 31 - 1, 66))])
def test_bad_rotations_are_rejected(kw):
    assert B.lib().mixkv_paged_append(C.byref(_params()), _caches(), _rows(), 1, C.byref(_rope(**kw)), 10, 1, None) == INVALID


def test_bad_sizes_are_rejected():
    p, L = C.byref(_params()), B.lib()
    for n_layers, n_rows, most in ((0, 10, 1), (129, 10, 1), (1, 0, 1), (1, 10, 0), (1, -4, 1)):
        assert L.mixkv_paged_append(p, _caches(), _rows(), n_layers, None, n_rows, most, None) == INVALID
        assert L.mixkv_paged_read(p, _caches(), _rows(), n_layers, n_rows, most, None) == INVALID
    assert L.mixkv_paged_append(p, None, _rows(), 1, None, 10, 1, None) == INVALID
    assert L.mixkv_paged_append(p, _caches(), None, 1, None, 10, 1, None) == INVALID
    assert L.mixkv_paged_read(p, _caches(), None, 1, 10, 1, None) == INVALID
    same = _rows(V=0x100000)
    assert L.mixkv_paged_read(p, _caches(), same, 1, 10, 1, None) == INVALID


@pytest.mark.parametrize("kw", [dict(Q=0), dict(Q=0x1008), dict(selected=0), dict(n_selected=0), dict(selected=0x2002), dict(n=0), dict(n=129), dict(null=True),
                                dict(keep=0), dict(keep=-1), dict(first=-1), dict(last=-1), dict(first=5, last=4), dict(first=2 ** 31 - 1, last=2 ** 31 - 1),
                                dict(ws=0), dict(ws=0x900010), dict(caches=_caches(K_bounds=0)), dict(caches=_caches(page_table=0))])
def test_bad_selections_are_rejected(kw):
    assert _select(**kw) == INVALID


@pytest.mark.parametrize("kw", [dict(Q=0), dict(Q=0x1008), dict(out=0), dict(out=0x2004), dict(selected=0), dict(n_selected=0), dict(selected=0x3001),
                                dict(n=0), dict(n=129), dict(null=True), dict(most=0), dict(most=1 << 25), dict(rows=0), dict(rows=-1),
                                dict(n=2, second=dict(selected=0, n_selected=0)), dict(caches=_caches(K_pages=0)), dict(caches=_caches(lengths=0))])
def test_bad_attention_arguments_are_rejected(kw):
    assert _attend(**kw) == INVALID


def test_workspaces():
    p = _params(max_pages=4096, n_pages=9000)
    n = B.mixkv_paged_select_workspace_size(p, 3)
    assert n % 256 == 0 and n >= 3 * 2 * 4 * 4096 * 4
    assert _select(p=p, n=3, size=n - 256) == B.MIXKV_ERR_WORKSPACE_TOO_SMALL
    L, size = B.lib(), C.c_size_t(0)
    assert L.mixkv_paged_select_workspace_size(C.byref(p), 0, C.byref(size)) == L.mixkv_paged_select_workspace_size(C.byref(p), 1, None) == INVALID
    for n_layers, rows in ((0, 100), (1, 0), (129, 1)):
        assert L.mixkv_paged_attention_workspace_size(C.byref(p), n_layers, rows, C.byref(size)) == INVALID
    assert L.mixkv_paged_attention_workspace_size(C.byref(p), 1, 1, None) == INVALID
    assert B.mixkv_paged_attention_workspace_size(p, 1, 32) == 0               # a tile is not split
    n = B.mixkv_paged_attention_workspace_size(p, 1, 200000)
    assert n % 256 == 0 and n > 0
    assert _attend(p=p, rows=200000, size=n - 256) == B.MIXKV_ERR_WORKSPACE_TOO_SMALL
    assert _attend(p=p, rows=200000, ws=0) == _attend(p=p, rows=200000, ws=0x900080) == INVALID
    # rows beyond what the table holds do not count
    assert B.mixkv_paged_attention_workspace_size(p, 1, 2 ** 31 - 1) == B.mixkv_paged_attention_workspace_size(p, 1, 4096 * 64)


def test_more_layers_and_heads_than_a_grid_are_refused():
    p = _params(batch=1, n_q_heads=1 << 18, n_kv_heads=1)            # 16384 groups of 16 query heads, in four layers
    assert _attend(p=p, n=4) == UNSUPPORTED


@pytest.mark.parametrize("scale", [2.0 ** 127 * 1.01, 2.9e38])
def test_scales_that_overflow_in_the_exponent_of_two_are_rejected(scale):
    with pytest.raises(B.MixkvError) as e:
        B.mixkv_page_bytes(_params(softmax_scale=scale))
    assert e.value.status == INVALID
    for fits in (2.0 ** 127, 1e-40):
        assert B.mixkv_page_bytes(_params(softmax_scale=fits)) > 0


@pytest.mark.parametrize("keep", [(1 << 24) + 1, 2 ** 31 - 1])
def test_selections_longer_than_any_table_are_rejected(keep):
    """As attention refuses such lists (64-row pages here): a thread's walk over 2^31 - 1 places would pass what 32 bits hold."""
    assert _select(keep=keep, first=0, last=0) == INVALID

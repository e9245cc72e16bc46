"""What a prepared paged call holds on to between its runs (no GPU: the calls are prepared over host tensors and never run)."""
import weakref

import pytest
import torch

from paper_2510_20707_amd import binding as B

P = dict(dtype="bf16", format="rows", batch=1, n_q_heads=4, n_kv_heads=2, head_dim=64, page_rows=32, max_pages=3, n_pages=5)
CPU = torch.device("cpu")


def _parts():
    p = B.make_paged_params(**P)
    t = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)  # noqa: E731
    i = lambda *shape: t(*shape, dtype=torch.int32)  # noqa: E731
    rows = B.PagedRows(t(6, 2, 64), t(6, 2, 64), i(1, 2), i(1, 2), t(6, 4, 64), t(6, 4, 64))
    rope = B.Rope(t(9, 32, dtype=torch.float32), t(9, 32, dtype=torch.float32), i(1, 6))
    return p, B.alloc_paged_cache(p, CPU, bounds=True), rows, rope, [t(1, 4, 64)], [t(1, 4, 64)], [i(1, 2, 2)], [i(1, 2)]


CALLS = {
    "append": lambda p, c, rows, rope, q, out, sel, n: B.PreparedPagedAppend(p, [c], [rows], rope),
    "read": lambda p, c, rows, rope, q, out, sel, n: B.PreparedPagedRead(p, [c], [rows]),
    "select": lambda p, c, rows, rope, q, out, sel, n: B.PreparedPagedSelect(p, [c], q, sel, n),
    "attention": lambda p, c, rows, rope, q, out, sel, n: B.PreparedPagedAttention(p, [c], q, out),
    "sparse": lambda p, c, rows, rope, q, out, sel, n: B.PreparedPagedAttention(p, [c], q, out, sel, n),
}
USES = {
    "append": ("K_pages", "V_pages", "page_table", "lengths", "K_bounds", "K", "V", "row_start", "row_count", "Q", "Q_out", "cos", "sin", "positions"),
    "read": ("K_pages", "V_pages", "page_table", "lengths", "K", "V", "row_start", "row_count"),
    "select": ("page_table", "lengths", "K_bounds", 4, 6, 7),
    "attention": ("K_pages", "V_pages", "page_table", "lengths", 4, 5),
    "sparse": ("K_pages", "V_pages", "page_table", "lengths", 4, 5, 6, 7),
}


@pytest.mark.parametrize("kind", list(CALLS))
def test_rebound_fields_leave_a_prepared_calls_tensors_alive(monkeypatch, kind):
    """A program that gives a field a new tensor (lengths + 1, a larger pool) does not free the one whose address the call has."""
    monkeypatch.setattr(B, "_paged_device", lambda caches: CPU)
    parts = _parts()
    call = CALLS[kind](*parts)
    refs = {}
    for name in USES[kind]:
        if isinstance(name, int):
            refs[name] = weakref.ref(parts[name][0])
            parts[name][0] = torch.zeros(1)
        else:
            owner = next(x for x in parts[1:4] if hasattr(x, name))
            refs[name] = weakref.ref(getattr(owner, name))
            setattr(owner, name, torch.zeros(1))
    assert [name for name, r in refs.items() if r() is None] == []
    del call
    assert [name for name, r in refs.items() if r() is not None] == []


@pytest.mark.parametrize("kind", list(CALLS))
def test_changed_params_do_not_reach_a_prepared_call(monkeypatch, kind):
    """The sizes that the buffers were checked against are those of every run."""
    monkeypatch.setattr(B, "_paged_device", lambda caches: CPU)
    parts = _parts()
    call = CALLS[kind](*parts)
    parts[0].batch, parts[0].n_pages, parts[0].max_pages = 7, 1000, 500
    given = call._args[0]._obj
    assert (given.batch, given.n_pages, given.max_pages) == (1, 5, 3)


def test_the_other_prepared_calls_hold_their_tensors():
    p = B.make_params("bf16", 1, 4, 2, 64, 40, 8, 10, budget_mode="adaptive")
    t = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)  # noqa: E731
    Ks, Vs, Qs, outs, ws = [t(1, 2, 40, 64)], [t(1, 2, 40, 64)], [t(1, 4, 8, 64)], [B.alloc_layer_out(p, CPU)], torch.zeros(1 << 10, dtype=torch.uint8)
    red, q, out, tails = [torch.zeros(1, 2)], [t(1, 4, 64)], [t(1, 4, 64)], [(t(1, 2, 3, 64), t(1, 2, 3, 64))]
    calls = [B.PreparedCall(p, Ks, Vs, Qs, outs, ws), B.PreparedDecode(p, outs, tails, q, out, 1), B.PreparedSimilarity(p, Ks, red, None, 8, ws)]
    refs = [weakref.ref(x) for x in (Ks[0], Vs[0], Qs[0], outs[0].K_out, outs[0].counts, outs[0].offsets, tails[0][0], tails[0][1], q[0], out[0], red[0])]
    for x in (Ks, Vs, Qs, red, q, out, tails):
        x[0] = None
    outs[0].K_out = outs[0].counts = outs[0].offsets = None
    assert all(r() is not None for r in refs)
    del calls
    assert all(r() is None for r in refs)

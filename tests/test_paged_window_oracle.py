"""The oracle of windows, weights and eviction, pinned by torch and by brute force (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from tests import newrows as R
from tests import paged as T


@pytest.mark.parametrize("fmt,dtype", [("rows", "f32"), ("4bit", "bf16")])
@pytest.mark.parametrize("window,first", [(R.ALL, 0), (5, 2), (1, 0), (9, 100)])
def test_window_attention_and_weights_against_torch(fmt, dtype, window, first):
    rng = np.random.default_rng(1)
    lay = T.Layer(rng, fmt, dtype, 64, 32, [[40, 23]], 2, fill=True)
    rows = R.Rows(rng, lay, 4, [12])
    out, lse = np.full(rows.Q.shape, 7.0), np.full(rows.Q.shape[:2], 7.0)
    O.window_attention(*rows.args(), window, first, 12, 0.5, out, lse)
    weights = rng.random((lay.n_pages, 32))
    before = weights.copy()
    O.window_weights(*rows.args(), window, first, 12, 0.5, lse, weights)
    for h, n in enumerate((40, 23)):
        k, v = (torch.from_numpy(x) for x in O.head(*lay.args(), lay.table, lay.lengths, 0, h))
        q = torch.from_numpy(rows.Q[:12, 2 * h:2 * h + 2])                           # [12, G, D]
        mask = torch.zeros(12, n, dtype=torch.bool)
        for t in range(12):
            for j in range(n):
                mask[t, j] = j <= n - 12 + t and (j > n - 12 + t - window or j < first)
        x = (0.5 * q @ k.T).masked_fill(~mask[:, None], -torch.inf)
        p = torch.softmax(x, -1)
        assert np.allclose(out[:12, 2 * h:2 * h + 2], p @ v, atol=1e-12) and np.allclose(lse[:12, 2 * h:2 * h + 2], torch.logsumexp(x, -1), atol=1e-12)
        for j in range(n):
            at = (lay.table[0, h, j // 32], j % 32)
            assert np.isclose(weights[at], (0.0 if j >= n - 12 else before[at]) + p[:, :, j].sum().item())
    assert (out[12:] == 7).all() and (lse[12:] == 7).all()


def test_rows_that_see_nothing():
    rng = np.random.default_rng(2)
    lay = T.Layer(rng, "rows", "bf16", 64, 32, [[3]], 2, fill=True)
    rows = R.Rows(rng, lay, 2, [5])                                                  # two rows more than the head has
    out, lse = np.full(rows.Q.shape, 7.0), np.full(rows.Q.shape[:2], 7.0)
    O.window_attention(*rows.args(), R.ALL, 0, 5, 1.0, out, lse)
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.isfinite(lse[2:5]).all()


def test_eviction_by_hand():
    w = np.array([5.0, 1.0, np.nan, 3.0, 3.0, -np.inf, 3.0, 0.0])
    there = np.ones(8, bool)
    assert O.evicted(w, there, 3, 0, 0) == [0, 3, 4] and O.evicted(w, there, 3, 0, 1) == [0, 3, 7] and O.evicted(w, there, 7, 0, 0) == [0, 1, 2, 3, 4, 6, 7]
    assert O.evicted(w, there, 2, 3, 3) == [0, 1] and O.evicted(w, there, 100, 0, 0) == list(range(8)) and O.evicted(w, there, -1, 2, 2) == []
    there[[0, 7]] = False
    assert O.evicted(w, there, 3, 1, 1) == [3, 4, 6]


@pytest.mark.parametrize("fmt,dtype,D,P", [("rows", "f32", 64, 32), ("rows", "bf16", 128, 32), ("4bit", "bf16", 64, 64), ("4bit", "bf16", 128, 32)])
@pytest.mark.parametrize("keys", [True, False])
def test_moved_rows_read_the_same(fmt, dtype, D, P, keys):
    rng = np.random.default_rng(3)
    src, dst = (rng.integers(0, 256, O.page_bytes(fmt, dtype, P, D), dtype=np.uint8) for _ in range(2))
    for r in range(P):
        for page in (src, dst):
            O.write_row(page, fmt, dtype, keys, P, r, O.as_dtype(rng.standard_normal(D), dtype))
    was, old = O.read_rows(src, fmt, dtype, keys, P, D), O.read_rows(dst, fmt, dtype, keys, P, D)
    O.move_row(src, 5, dst, P - 3, fmt, dtype, keys, P, D)
    now = O.read_rows(dst, fmt, dtype, keys, P, D)
    assert np.array_equal(now[P - 3], was[5]) and np.array_equal(np.delete(now, P - 3, 0), np.delete(old, P - 3, 0))

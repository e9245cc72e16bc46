"""Launches and workspaces of the calls on pages at the ends of what they accept (no GPU; tests/launches.py): a launch has fewer than 2^32 threads and at most 65535 workgroups along y and z."""
import ctypes as C
import itertools
import math

import pytest

from paper_2510_20707_amd import binding as B
from tests import launches
from tests import test_paged_window_abi as W

# (batch, query heads, KV heads): one sequence, and the most that a call takes, in heads and in sequences
SHAPES = [(1, 28, 4), (64, 32, 8), (4096, 8, 8), (512, 512, 8), (1, 1 << 18, 1 << 18), (1 << 18, 1, 1)]
KINDS = [("rows", "bf16"), ("4bit", "bf16"), ("rows", "f32")]


def _params(shape, kind):
    batch, hq, hkv = shape
    return dict(format=kind[0], dtype=kind[1], batch=batch, n_q_heads=hq, n_kv_heads=hkv, page_rows=64, max_pages=1 << 24, n_pages=40)


def _check(calls, tmp_path, most_bytes=None):
    made = 0
    for call, (status, need, launched) in zip(calls, launches.record(calls, tmp_path)):
        assert status == 0 and launched, call
        assert most_bytes is None or need <= most_bytes, (need, call)
        for name, grid, block in launched:
            assert min(grid) > 0 and max(grid[1:]) <= 65535 and math.prod(grid) * math.prod(block) < 1 << 32, (name, grid, block, call)
        made += len(launched)
    assert made >= len(calls)


@pytest.mark.parametrize("shape", SHAPES)
def test_weights(shape, tmp_path):
    """One long prompt among many short sequences, windows short and long, first rows that every row sees: the sums of chunks are those of at most 16384 blocks of 512 keys, and of
    65536 blocks of first keys."""
    calls = []
    for kind, layers, rows, count in itertools.product(KINDS, (1, 24, 128), (1000, 163840, 1 << 30), (1, 1000, 163840)):
        if (kind[1] == "f32" and count > 1000) or count * shape[1] >= 1 << 31:
            continue
        calls += [("weigh", _params(shape, kind), dict(n=layers, rows=count, window=window, first=first, count=count, most=rows))
                  for window, first in ((1 << 30, 0), (64, 16), (64, 100000), (1, 1 << 30))]
    _check(calls, tmp_path, (16384 + 65536) * 512 * 4)


@pytest.mark.parametrize("shape", SHAPES)
def test_eviction(shape, tmp_path):
    _check([("evict", _params(shape, kind), dict(n=layers, keep=rows, rows=rows))
            for kind, layers, rows in itertools.product(KINDS, (1, 16, 24, 128), (1, 1000, 4096, 16384, 163840, 1 << 30))], tmp_path)


@pytest.mark.parametrize("shape", SHAPES)
def test_attention(shape, tmp_path):
    """Few rows of the most heads, many of a few."""
    calls = []
    for kind, layers, rows, count in itertools.product(KINDS, (1, 24, 128), (1000, 163840, 1 << 30), (1, 5, 64, 163840)):
        if count * math.prod(shape[:2]) * layers > 1 << 26 or count * shape[1] >= 1 << 31:
            continue
        calls += [("attend", _params(shape, kind), dict(n=layers, rows=count, window=window, first=first, count=count, most=rows)) for window, first in ((1 << 30, 0), (64, 16), (64, 100000))]
    _check(calls, tmp_path)


@pytest.mark.parametrize("shape", SHAPES)
def test_selection_and_single_tokens(shape, tmp_path):
    """Tables of few pages and of the most (attention refuses more groups of query heads than a launch has places for)."""
    calls = []
    for kind, layers, pages in itertools.product(KINDS, (1, 16, 32, 128), (16, 4097, 1 << 24)):
        p = dict(_params(shape, kind), max_pages=pages)
        calls += [("select", p, dict(n=layers))] + [("single", p, dict(n=layers, rows=rows)) for rows in (1000, 1 << 30) if shape[1] // shape[2] <= 1 << 14]
    _check(calls, tmp_path)


def test_rows_that_32_bits_do_not_count():
    """Chunks of rows that a block of keys does not have, and the turns behind a unit's last row, stay below 2^31: weights take up to 2^30 rows times query heads."""
    for hq, hkv in ((1, 1), (28, 4), (8, 1), (1 << 18, 1)):
        p, need = W._params(n_q_heads=hq, n_kv_heads=hkv, batch=1, format="rows"), C.c_size_t()
        most = (1 << 30) // hq
        size = lambda rows: B.lib().mixkv_paged_weights_workspace_size(C.byref(p), 1, rows, 1 << 30, 0, rows, 1 << 20, C.byref(need))  # noqa: E731
        assert size(most) == B.MIXKV_OK and size(most + 1) == size((2 ** 31 - 1) // hq) == B.MIXKV_ERR_UNSUPPORTED
        assert W._weigh(p, rows=most + 1, count=most + 1) == B.MIXKV_ERR_UNSUPPORTED

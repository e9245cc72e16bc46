"""mixkv_paged_window_attention and mixkv_paged_weights where a wide tolerance would hide what they are built for: logits of 4-bit pages in full, the same log-sum-exp whatever the kernel, tiles without any
weight, and chunks of rows that many heads share."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2510_20707_amd import binding as B
from tests import newrows as R
from tests import newrows4 as X
from tests import paged as T

pytestmark = pytest.mark.gpu
KINDS = [("rows", "f32"), ("rows", "bf16"), ("4bit", "bf16")]


@pytest.mark.parametrize("D,P", [(128, 64), (64, 32), (128, 32), (64, 128)])
@pytest.mark.parametrize("count", [1, 5, 80])
def test_4bit_keys_and_query_sums_count_in_full(D, P, count):
    """The limits that tests/test_paged_window_bounds.py shows a single fp16 part to exceed four times over."""
    print(f"[case] full 4bit D={D} P={P} count={count}", flush=True)
    rng = np.random.default_rng([91, D, P, count])
    rows = X.make(rng, D, P, [[200, 171]], 3, [count])
    lay, scale = rows.lay, 0.125
    for window, first in ((R.ALL, 0), (50, 10)):
        q = R.attend(rows, window, first, scale)
        out, lse = R.check_attention(rows, q, window, first, scale)
        got = q.lse.cpu().numpy().astype(np.float64)
        off = np.abs(got - lse)[:count]
        assert (off <= X.lse_limit(rows, scale, lse)[:count]).all(), float(off.max())
        # the weights against the oracle's normaliser
        before = rng.random((lay.n_pages, lay.P)).astype(np.float32)
        w = torch.from_numpy(before.copy()).to(T.DEV)
        q.lse.copy_(torch.from_numpy(lse.astype(np.float32)))
        B.mixkv_paged_weights(lay.params(rows.hq, scale), [lay.device()], [q], [w], window, first, max_count=count)
        want = before.astype(np.float64)
        O.window_weights(*rows.args(), window, first, count, scale, lse.astype(np.float32).astype(np.float64), want)
        rel = np.abs(w.cpu().numpy() - want) / np.maximum(want, 1e-30)
        print(f"       lse off by {off.max():.2e}, weights by {rel.max():.2e}", flush=True)
        assert (rel <= X.weight_limit(rows, scale)).all(), float(rel.max())


@pytest.mark.parametrize("fmt,dtype", KINDS)
def test_the_same_log_sum_exp_whatever_the_kernel(fmt, dtype):
    """A prompt's rows together, six at a time and one at a time: each log-sum-exp within the oracle's limit (tests/newrows.py), any two within twice that."""
    rng = np.random.default_rng(69)
    lay = T.Layer(rng, fmt, dtype, 64, 32, [[140, 140]], 5, fill=True)
    rows = R.Rows(rng, lay, 6, [140], pad=0)
    whole = R.attend(rows, 33, 4)
    R.check_attention(rows, whole, 33, 4)
    limit = 2 * (rows.logit_error(1.0) + 4 * 2.0 ** -24 * (1 + float(whole.lse.abs().max())) + 2.0 ** -20)
    assert limit <= (6e-3 if fmt == "4bit" else 3e-4)
    for count, ends in ((1, (0, 31, 32, 36, 37, 139)), (6, (5, 32, 40, 139))):
        few = R.Rows(rng, lay, 6, [count], pad=0)
        for t in ends:
            lay.lengths[:] = t + 1
            few.Q = rows.Q[t + 1 - count:t + 1]
            q = R.attend(few, 33, 4)
            R.check_attention(few, q, 33, 4)
            off = (q.lse - whole.lse[t + 1 - count:t + 1]).abs().max()
            assert float(off) <= limit, (count, t, float(off))
            lay.lengths[:] = 140


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,P", [(128, 32), (64, 64)])
@pytest.mark.parametrize("count", [1, 5, 80])
def test_tiles_without_weight_within_the_oracles_tolerance(dtype, D, P, count):
    """Keys of minus infinity: whole tiles, whole windows, everything: outputs and finite log-sum-exps by the limits of tests/newrows.py."""
    rng = np.random.default_rng([92, D, count])
    n = 300
    lay = T.Layer(rng, "rows", dtype, D, P, [[n]], -(-n // P), fill=True)
    rows = R.Rows(rng, lay, 5, [count])
    rows.Q[..., 7] = O.as_dtype(np.abs(rows.Q[..., 7]) + 0.5, dtype)
    i = np.arange(n)
    for off in (i // 32 % 3 != 1, i // 32 % 2 == 0, i < n - 3, i < n - 90, np.ones(n, bool)):
        for r in range(n):
            page = lay.K[lay.table[0, 0, r // P]]
            row = O.read_rows(page, "rows", dtype, True, P, D)[r % P]
            row[7] = -np.inf if off[r] else 0.25
            O.write_row(page, "rows", dtype, True, P, r % P, row)
        for window, first in ((R.ALL, 0), (40, 20)):
            out, lse = R.check_attention(rows, R.attend(rows, window, first), window, first)
            assert (out[np.isneginf(lse)] == 0).all() and (off.all() or np.isfinite(lse).any())


@pytest.mark.parametrize("fmt,dtype", [("rows", "bf16"), ("4bit", "bf16")])
@pytest.mark.parametrize("batch", [6000, 70000])
def test_first_keys_of_many_heads(fmt, dtype, batch):
    """One prompt of 7000 rows beside thousands of sequences, of which a few have a token and the others none: the chunks of the rows that see the first keys are those that the heads leave, ten or
    none of their own."""
    print(f"[case] first keys {fmt} {batch}", flush=True)
    rng = np.random.default_rng(93)
    n, P = 7000, 128
    lens = np.zeros((batch, 1), np.int32)
    lens[17], lens[18:40] = n, rng.integers(1, 300, (22, 1))
    lay = T.Layer(rng, fmt, dtype, 64, P, lens, -(-n // P), fill=True)
    rows = R.Rows(rng, lay, 2, np.where(lens == n, n, np.minimum(lens, 1)))
    q = R.attend(rows, 8, 1)
    R.check_attention(rows, q, 8, 1)
    before = rng.random((lay.n_pages, P)).astype(np.float32)
    got = []
    for _ in range(2):
        w = torch.from_numpy(before.copy()).to(T.DEV)
        B.mixkv_paged_weights(lay.params(2), [lay.device()], [q], [w], 8, 1, max_count=n)
        got.append(w.cpu().numpy())
    R.check_weights(rows, q.lse.cpu().numpy(), before, got[0], 8, 1)
    assert np.array_equal(*got)                                                      # repeated bit for bit

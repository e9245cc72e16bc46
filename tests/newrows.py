"""New rows of queries on a test layer (tests/paged.py): their buffers on host and device, and the comparison with the oracle."""
import numpy as np
import torch

from oracle import paged_oracle as O
from paper_2510_20707_amd import binding as B
from tests import paged as T

ALL = B.EVERY_ROW
MANY = 64                                     # rows of a unit (new rows times query heads) above which rows go through the kernels of prompts


class Rows:
    """Ragged queries: per sequence `counts` rows one after another (pad unused ones behind them), the same for all its heads unless counts is [batch, Hkv]."""

    def __init__(self, rng, lay, hq, counts, pad=3, spread=2.0, start=None):
        batch, hkv = lay.lengths.shape
        self.lay, self.hq, self.G = lay, hq, hq // hkv
        self.count = np.broadcast_to(np.asarray(counts, np.int32).reshape(batch, -1), (batch, hkv)).copy()
        most = np.maximum(self.count.max(1), 0)
        first = (np.cumsum(most) - most).astype(np.int32)
        self.start = np.repeat(first[:, None], hkv, 1) if start is None else np.asarray(start, np.int32)
        self.n = int(most.sum()) + pad
        self.Q = O.as_dtype(rng.standard_normal((self.n, hq, lay.D)) * spread / np.sqrt(lay.D), lay.dtype)
        self.max_count = int(max(most.max(), 1))

    def device(self, strided=False):
        """(queries, outputs full of 7, lse full of 7); strided: Q is part of a larger tensor."""
        q = T.to_device(self.Q, self.lay.dtype)
        if strided:
            big = torch.full((self.n, self.hq + 5, self.lay.D), 3.0, dtype=q.dtype, device=T.DEV)
            big[:, 2:2 + self.hq] = q
            q = big[:, 2:2 + self.hq]
        out = torch.full((self.n, self.hq, self.lay.D), 7.0, dtype=q.dtype, device=T.DEV)
        return B.PagedQueries(q, T.i32(self.start), T.i32(self.count), out, torch.full((self.n, self.hq), 7.0, device=T.DEV))

    def args(self):
        return self.lay.args(), self.lay.table, self.lay.lengths, self.Q, self.start, self.count

    def logit_error(self, scale):
        """How far a logit may be off: a fp32 sum of D terms by D 2^-24 of their magnitudes' sum (4-bit keys are summed as S sum(q u) + B sum(q), or in two fp16
        parts, with terms of up to 8 max |k| |q|)."""
        most = 0.0
        for b, h in np.ndindex(*self.lay.lengths.shape):
            k, _, there = O.rows_of(*self.lay.args(), self.lay.table, self.lay.lengths, b, h)
            k = k[there & np.isfinite(k).all(1)]
            if len(k):
                q = np.abs(self.Q[:, h * self.G:(h + 1) * self.G])
                most = max(most, float(q.sum(-1).max() * 8 * np.abs(k).max()) if self.lay.fmt == "4bit" else float((q.reshape(-1, self.lay.D) @ np.abs(k).T).max()))
        return self.lay.D * 2.0 ** -24 * most * scale


def attend(rows, window=ALL, first=0, scale=1.0, max_count=None, max_rows=None, strided=False, cache=None):
    cache, q = cache or rows.lay.device(), rows.device(strided)
    B.mixkv_paged_window_attention(rows.lay.params(rows.hq, scale), [cache], [q], window, first, max_count=max_count or rows.max_count, max_rows=max_rows)
    return q


def check_attention(rows, q, window=ALL, first=0, scale=1.0, max_count=None):
    """Per output row: |gpu - oracle| <= tol max_d |oracle_d| + more * max |v|.
      f32   tol 1e-5: fp32 accumulation, as for the single token's attention; bf16 2^-8 + 1e-4: the output's rounding and the fp32 sums before it
      more  2 * the logits' error (weights off by a factor e^+-d move the output by 2 d max |v|); 4bit: 2 * 2^-11 beside it for values and weights in fp16;
            bf16 of many rows: 2^-8, the rounding of the weights (of the numerators; the sum that divides them takes them unrounded)
    lse: the logits' error, and fp32 roundings of the offset, its logarithm and their sum, 4 * 2^-24 of (1 + |lse|), and 2^-20 for the sum of weights under the logarithm."""
    lay = rows.lay
    lay_v = max((float(np.abs(v[np.isfinite(v)]).max(initial=0.0)) for v in (O.rows_of(*lay.args(), lay.table, lay.lengths, b, h)[1] for b, h in np.ndindex(*lay.lengths.shape))), default=0.0)
    coarse = min(rows.max_count, max_count or rows.max_count) * rows.G > MANY
    d = rows.logit_error(scale)
    out, lse = np.full(rows.Q.shape, 7.0), np.full(rows.Q.shape[:2], 7.0)
    with np.errstate(invalid="ignore"):
        O.window_attention(*rows.args(), window, first, max_count or rows.max_count, scale, out, lse)
    got, sums = T.values(q.out), q.lse.cpu().numpy().astype(np.float64)
    tol = 1e-5 if lay.dtype == "f32" else 2.0 ** -8 + 1e-4
    more = 2 * d + (2 * 2.0 ** -11 if lay.fmt == "4bit" else 2.0 ** -8 if coarse and lay.dtype == "bf16" else 0.0)
    fine = np.isfinite(out)
    # (Values are to stay below 2^100.  A row that sees an infinity has no number there, but whether an infinity or a NaN is not said: bf16 weights are
    # taken in two parts, of which the second may be zero or negative, and its product with an infinity decides.)
    assert np.array_equal(np.isfinite(got), fine)
    err = np.abs(np.where(fine, got - np.where(fine, out, 0.0), 0.0)).max(-1)
    limit = tol * np.abs(np.where(fine, out, 0.0)).max(-1) + more * lay_v
    kept = (out == 7.0).all(-1)
    assert (err <= np.where(kept, 0.0, limit)).all(), (float((err / np.maximum(limit, 1e-30)).max()), np.argwhere(err > limit)[:5].tolist())
    same = np.isneginf(lse)
    assert np.array_equal(np.isneginf(sums), same)
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0.0, np.abs(sums - lse))
    assert (off <= d + 4 * 2.0 ** -24 * (1 + np.abs(np.where(same, 0.0, lse))) + 2.0 ** -20).all(), float(off.max())
    print(f"       {float((err / np.maximum(limit, 1e-30)).max()):.3f} of the tolerance", flush=True)
    return out, lse


def check_weights(rows, lse, before, got, window=ALL, first=0, scale=1.0, max_count=None):
    """|gpu - oracle| <= oracle * (2 d + 2^-16): the logits' error, the normaliser's and the exponent's roundings (2^-23 of magnitudes up to some 2^5), the sum's (2^-18)."""
    lay = rows.lay
    want = before.astype(np.float64).copy()
    O.window_weights(*rows.args(), window, first, max_count or rows.max_count, scale, lse.astype(np.float64), want)
    d = rows.logit_error(scale)
    same = np.isnan(want)
    assert np.array_equal(np.isnan(got), same)
    err = np.where(same, 0.0, np.abs(got - want))
    assert (err <= np.where(same, 0.0, np.abs(want)) * (2 * d + 2.0 ** -16) + 1e-30).all(), float(np.nanmax(err / (np.abs(want) + 1e-30)))
    assert np.array_equal(got[want == before], before[want == before])
    print(f"       weights off by {float(np.nanmax(err / (np.abs(want) + 1e-30))):.2e}", flush=True)

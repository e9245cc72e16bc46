"""New rows on 4-bit pages whose logits show each rounding to fp16 that the kernels go out of their way to avoid, and how far log-sum-exp and weights may then be off.

Keys are 1 + S (1 + code / 16) with S of 0.9 halves of fp16's step behind 1 and codes 0 and 1: rounded to fp16 every element is 1, off by 0.9 to 0.957 times 2^-11, all to one side.  Queries are
one but for an element of 1 + 2^-7 in each group of 32, whose sum of 32 + 2^-7 is 32 in fp16, off by 2^-12 of it.  Every term of a logit is positive, so the roundings of fp32 stay in proportion to it."""
import numpy as np

from oracle import paged_oracle as O
from tests import newrows as R
from tests import paged as T

STEP, BASE = np.float16(0.9 * 2.0 ** -11), np.float16(1.0)


def make(rng, D, P, lens, G, counts):
    lay = T.Layer(rng, "4bit", "bf16", D, P, lens, -(-int(np.max(lens)) // P), fill=True)
    for page in lay.K:
        words, halves = page[:P * D // 2].view(np.uint32), page[P * D // 2:].view(np.float16)
        words[:] = rng.integers(0, 2 ** 32, len(words), dtype=np.uint32) & 0x11111111
        halves[0::2], halves[1::2] = STEP, BASE
    rows = R.Rows(rng, lay, lay.lengths.shape[1] * G, counts)
    rows.Q = np.ones_like(rows.Q)
    at = rng.integers(0, 32, rows.Q.shape[:2] + (D // 32,)) + 32 * np.arange(D // 32)
    np.put_along_axis(rows.Q, at, 1 + 2.0 ** -7, 2)
    rows.Q *= 2.0 ** -(np.arange(rows.hq) % G)[:, None]
    return rows


def logit_error(rows, scale):
    """A product's sum over D elements in two parts is 2 D additions (in 16-element steps a kernel makes fewer); the codes' own share is 2^-11 of a logit.  48 more: the query sums (9 additions), their
    products with steps and bases (24), the groups' sums (4), the scale, and what two fp16 parts of a key and three of a sum leave out (2^-22)."""
    D = rows.lay.D
    return scale * (2 * D + 48) * 2.0 ** -24 * np.abs(rows.Q).sum(-1).max() * (1 + 2 * float(STEP))


def lse_limit(rows, scale, lse):
    """The logits' error, the offset, its logarithm and their sum, and the additions of the weights of up to n rows."""
    n = int(rows.lay.lengths.max())
    return logit_error(rows, scale) + 4 * 2.0 ** -24 * (1 + np.abs(lse)) + (n + 8) * 2.0 ** -24


def weight_limit(rows, scale):
    """Relative: the logit's error, the exponent's roundings (of magnitudes up to twice the logit, normaliser and scale constants, the exponential itself) and the additions of one weight a row."""
    top = scale * np.abs(rows.Q).sum(-1).max() * 1.01
    return logit_error(rows, scale) + 8 * 2.0 ** -24 * (2 + 2 * top) + (int(rows.count.max()) * rows.G + 8) * 2.0 ** -24


def emulated(rows, b, h, key_parts, sum_parts, scale, window, first):
    """Log-sum-exp of a head's rows [served, G] in 64 bits but for one rounding: keys, or the queries' sums of a group, in one fp16 part."""
    lay, D = rows.lay, rows.lay.D
    k, _, there = O.rows_of(*lay.args(), lay.table, lay.lengths, b, h)
    assert there.all()
    if key_parts == 1:
        k = k.astype(np.float16).astype(np.float64)
    out = []
    for row, place in O.new_rows(lay.lengths, rows.start, rows.count, b, h, len(k), rows.n, rows.max_count):
        q = rows.Q[row, h * rows.G:(h + 1) * rows.G]
        x = q @ k.T
        if sum_parts == 1:
            sums = q.reshape(rows.G, D // 32, 32).sum(-1)
            x += ((sums.astype(np.float16).astype(np.float64) - sums) * (float(BASE) + float(STEP))).sum(-1, keepdims=True)
        x = np.where(O.sees(place, len(k), window, first), scale * x, -np.inf)
        top = x.max(1)
        out.append(top + np.log(np.exp(x - top[:, None]).sum(1)))
    return np.array(out)


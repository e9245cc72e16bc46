"""What the bounds of tests/newrows4.py would see (no GPU): a kernel that kept keys, or the queries' sums, in one fp16 part would be off by more than they allow, and without either it is not."""
import numpy as np
import pytest

from oracle import paged_oracle as O
from tests import newrows as R
from tests import newrows4 as X


@pytest.mark.parametrize("D,P", [(128, 64), (64, 32), (128, 32), (64, 128)])
@pytest.mark.parametrize("count", [1, 5, 80])
def test_one_part_is_off_by_more_than_the_bounds(D, P, count):
    rng = np.random.default_rng([91, D, P, count])
    rows = X.make(rng, D, P, [[200, 171]], 3, [count])
    for window, first in ((R.ALL, 0), (50, 10)):
        out, lse = np.zeros(rows.Q.shape), np.zeros(rows.Q.shape[:2])
        O.window_attention(*rows.args(), window, first, rows.max_count, 0.125, out, lse)
        for h in range(2):
            want = lse[:count, 3 * h:3 * h + 3]
            limit = X.lse_limit(rows, 0.125, want)
            both = X.emulated(rows, 0, h, 2, 3, 0.125, window, first)
            assert np.abs(both - want).max() <= 1e-9
            for parts in ((1, 3), (2, 1)):
                off = np.abs(X.emulated(rows, 0, h, *parts, 0.125, window, first) - want)
                # of the largest head: the limit is the launch's, a smaller head's logits are a half and a quarter
                assert (off[:, 0] > 4 * limit[:, 0]).all(), (parts, float(off[:, 0].min()), float(limit.max()))
                assert (off[:, 0] > 4 * X.weight_limit(rows, 0.125)).all()     # against a normaliser in 64 bits a weight is off by as much, relatively

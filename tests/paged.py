"""Paged caches for tests: random ones on the host with the buffers of one layer, their copies on the device."""
import numpy as np
import torch

from oracle import paged_oracle as O
from paper_2510_20707_amd import binding as B

DEV = "cuda:0"


def to_device(x, dtype):
    """Float64 values of the dtype -> device tensor (NaN and infinities kept)."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(B.TORCH_DTYPE[B.DTYPE[dtype]]).to(DEV)


def values(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Layer:
    """One layer's cache: pools of random bytes, a page table of distinct pages, host and device copies."""

    def __init__(self, rng, fmt, dtype, D, P, lengths, max_pages, spare=2, bounds=False, fill=False):
        self.fmt, self.dtype, self.D, self.P = fmt, dtype, D, P
        self.lengths = np.asarray(lengths, np.int32)
        units = self.lengths.size
        need = np.minimum(-(-np.maximum(self.lengths, 0) // P), max_pages)
        self.n_pages = int(need.sum()) + spare
        self.table = np.full(self.lengths.shape + (max_pages,), -1, np.int32)
        ids = rng.permutation(self.n_pages)
        flat, at = self.table.reshape(units, max_pages), 0
        for u in range(units):
            n = int(need.reshape(-1)[u])
            flat[u, :n] = ids[at:at + n]
            at += n
        size = O.page_bytes(fmt, dtype, P, D)
        self.K, self.V = (rng.integers(0, 256, (self.n_pages, size), dtype=np.uint8) for _ in range(2))
        self.bounds = O.as_dtype(rng.standard_normal((self.n_pages, 2, D)), dtype) if bounds else None
        if fill:                                  # rows that a program has written before
            for b, h in np.ndindex(*self.lengths.shape):
                mean = rng.standard_normal(D)
                for r in range(min(max(int(self.lengths[b, h]), 0), max_pages * P)):
                    page = self.table[b, h, r // P]
                    O.write_row(self.K[page], fmt, dtype, True, P, r % P, O.as_dtype(rng.standard_normal(D) + mean, dtype))
                    O.write_row(self.V[page], fmt, dtype, False, P, r % P, O.as_dtype(rng.standard_normal(D), dtype))

    def args(self):
        return self.fmt, self.dtype, self.P, self.D, self.K, self.V

    def device(self):
        t = lambda x: torch.from_numpy(x.copy()).to(DEV)  # noqa: E731
        return B.PagedCache(t(self.K), t(self.V), t(self.table), t(self.lengths), None if self.bounds is None else to_device(self.bounds, self.dtype))

    def params(self, hq, scale=1.0):
        return B.make_paged_params(self.dtype, self.fmt, self.lengths.shape[0], hq, self.lengths.shape[1], self.D, self.P, self.table.shape[2],
                                   self.n_pages, scale)


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)

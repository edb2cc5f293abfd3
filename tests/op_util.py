"""Inputs and checks shared by the cache's tests (no test functions here)."""
import numpy as np
import torch

import paper_2604_20819_amd as cq
from oracle import cache4 as o4

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {k: torch.finfo(v).eps / 2 for k, v in DT.items()}


def normal(g, shape, dtype):
    return torch.from_numpy(g.standard_normal(shape, dtype=np.float32)).to(DT[dtype])


class Case:
    """Sequences of `lens` tokens in a pool of pages in any order, with spare pages; the
    pool starts as `fill` in every byte."""

    def __init__(self, seed, lens, H, d, page, fill=0xFF, spare=2, extra_columns=1):
        self.g = np.random.Generator(np.random.PCG64(seed))
        self.lens, self.H, self.d, self.page = list(lens), H, d, page
        need = [-(-n // page) for n in lens]
        self.n_pages = sum(need) + spare
        order = self.g.permutation(self.n_pages)
        self.table = np.full((len(lens), max(need + [0]) + extra_columns), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.data = np.full((self.n_pages, o4.page_bytes(page, H, d)), fill, np.uint8)

    def slots(self, b, first, n):
        """Pages (-1: none) and tokens of sequence b's positions first ... first + n - 1."""
        pos = np.arange(first, first + n)
        ok = (pos >= 0) & (pos // self.page < self.table.shape[1])
        p = np.where(ok, self.table[b, np.where(ok, pos // self.page, 0)], -1)
        return p, np.where(pos >= 0, pos, 0) % self.page

    def fill_tokens(self, gain=1.0):
        """Every sequence's tokens written (by the oracle); returns k, v per sequence."""
        out = []
        for b, n in enumerate(self.lens):
            k = self.g.standard_normal((n, self.H, self.d)) * gain
            k[..., 5::13] *= 4
            v = self.g.standard_normal((n, self.H, self.d))
            p, t = self.slots(b, 0, n)
            o4.write(self.data, self.page, k, v, p, t)
            out.append((k, v))
        return out

    def cache(self, device="cuda"):
        return cq.Cache4(self.n_pages, self.H, self.d, page_size=self.page,
                         data=torch.from_numpy(self.data.copy()).to(device))

    def batch(self, lens=None, **kw):
        return cq.CacheBatch(torch.from_numpy(self.table).cuda(),
                             torch.tensor(self.lens if lens is None else lens, dtype=torch.int32, device="cuda"), **kw)


def starts(new, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(new)]).astype(np.int32)).cuda()


# Calls of cqsa_cache_weigh whose waves go through several tiles of tokens, one after the other: sequences, heads,
# query heads a head, rows, d, dtype, the longest sequence.
WEIGH_LOOPS = [
    (16, 16, 1, 1, 32, "bf16", 4100), (3, 64, 8, 2, 128, "f16", 3001), (2, 64, 5, 6, 128, "bf16", 5000),
    (2, 96, 3, 4, 96, "f32", 2777), (1, 256, 1, 1, 32, "bf16", 50003),  # few rows; more than 64 tiles
    (8, 64, 5, 9, 64, "bf16", 3000), (5, 96, 1, 100, 96, "f16", 2100), (4, 64, 4, 12, 256, "f32", 3100),  # rows that stay
]

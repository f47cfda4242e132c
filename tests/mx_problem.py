"""Problems for the operators of hyp_mx.h: a cache written by mx_write, and what the reference says of it."""
from __future__ import annotations

import torch

import paper_2511_14450_amd as hyp
from tests import mx_reference as ref

BF, F32 = torch.bfloat16, torch.float32


class Problem:
    """Requests of `held` keys, whose first `held - rows` were written before; everything on the host, and the cache on the device.

    layout  "slab", "pages" (shuffled, more of them than are named), "inner" (slabs with the heads inside the keys, tensors with gaps)
    """

    def __init__(self, seed, held, nkv=2, d=64, formats=("e4m3", "e2m1"), block=16, layout="slab", page=32, dtype=F32, spread=1.0, most=None):
        self.gen = torch.Generator().manual_seed(seed)
        self.held, self.nkv, self.d, self.formats, self.block, self.dtype = list(held), nkv, d, formats, block, dtype
        n, groups, unit = len(held), -(-d // 32), max(block, 16)
        self.most = max(max(held), 1) if most is None else most
        widths = [ref.FORMATS[f]["bytes"] * groups for f in formats]
        table = None
        if layout == "pages":
            per = -(-self.most // page)
            table = torch.randperm(n * per + 3, generator=self.gen)[:n * per].reshape(n, per).int()
            slabs, room = n * per + 3, page
        else:
            slabs, room = n, -(-self.most // unit) * unit
        byte = lambda *shape: torch.randint(0, 256, shape, generator=self.gen, dtype=torch.uint8).cuda()  # what no key has written holds anything, NaN too  # noqa: E731
        if layout == "inner":
            self.k, self.v = (byte(slabs, room, nkv, w + 16)[..., :w].transpose(1, 2) for w in widths)
            self.ks, self.vs = (byte(slabs, groups, nkv, room + 4)[..., :room].transpose(1, 2) for _ in widths)
        else:
            self.k, self.v = (byte(slabs, nkv, room, w) for w in widths)
            self.ks, self.vs = (byte(slabs, nkv, groups, room) for _ in widths)
        self.lo = self.hi = None
        if block:
            shape = (slabs, nkv, room // block, d)
            self.lo, self.hi = (torch.full(shape, float("nan"), dtype=BF, device="cuda") for _ in range(2))
            if layout == "inner":
                self.lo, self.hi = (torch.full((slabs, room // block, nkv, d + 3), float("nan"), dtype=BF, device="cuda")[..., :d].transpose(1, 2) for _ in range(2))
        self.table = table
        self.lens = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.cache = hyp.MxCache(self.k, self.v, self.ks, self.vs, self.lens, d, page_table=None if table is None else table.cuda(), most=self.most, lo=self.lo, hi=self.hi)
        # rows of every request, and the numbers that the formats hold of them
        self.rows_k = [(torch.randn((h, nkv, d), generator=self.gen) * spread).to(dtype) for h in held]
        self.rows_v = [torch.randn((h, nkv, d), generator=self.gen).to(dtype) for h in held]

    def values(self):
        """Numbers of all keys [held, heads, d] a request, in 64 bits"""
        return [[ref.stored_rows(f, x) for x in rows] for f, rows in zip(self.formats, (self.rows_k, self.rows_v))]

    def write(self, first, last, single=False, **more):
        """Keys first[b] .. last[b] - 1 of every request, as one call"""
        self.lens.copy_(torch.tensor(last, dtype=torch.int32))
        k, v = (torch.cat([x[a:z] for x, a, z in zip(rows, first, last)]).cuda() for rows in (self.rows_k, self.rows_v))
        start = None
        if not single:
            counts = [z - a for a, z in zip(first, last)]
            start = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32).cuda()
        hyp.mx_write(self.cache, k, v, q_start=start, **more)
        return k, v

    def fill(self):
        self.write([0] * len(self.held), self.held)
        return self

    def place(self, b, j, per):
        if self.table is None:
            return b, j
        return int(self.table[b, j // per]), j % per

    def codes(self, b, c, j):
        """(numbers of key j, of its value) by their codes"""
        page, at = self.place(b, j, self.k.shape[2])
        return [torch.tensor(ref.codes(f, x[page, c, at].tolist(), s[page, c, :, at].tolist())[:self.d], dtype=torch.float64)
                for f, x, s in zip(self.formats, (self.k, self.v), (self.ks, self.vs))]

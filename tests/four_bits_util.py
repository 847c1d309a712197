"""A paged cache in 4 bits for the tests, from the documented layout; shares no code with the library."""
from __future__ import annotations

import torch

import paper_2512_17970_amd as cg
from gpu_util import Guarded


def bit_of(j):
    return 4 * (j // 2) + 16 * (j % 2)


def unpack(words):
    """The eight codes of each word, in order."""
    w = words.long() & 0xFFFFFFFF
    return torch.stack([(w >> bit_of(j)) & 15 for j in range(8)], dim=-1)


def pack(codes):
    """[..][8] -> words"""
    w = sum(codes[..., j].long() << bit_of(j) for j in range(8))
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


class Cache4:
    """Between canary bands; scales and offsets of places that hold no token are NaN, their codes anything."""

    def __init__(self, lens, *, heads=2, dim=64, page=16, block=32, seed=0, spare=3, max_pages=None, filled=None, quick=False):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.heads, self.dim, self.page, self.block = list(lens), heads, dim, page, block
        self.runs, self.dtype = -(-dim // block), cg.KV_INT4
        used = [-(-max(n, 0) // page) for n in lens]
        if max_pages:
            used = [min(n, max_pages) for n in used]
        self.max_pages = max_pages or max(1, max(used))
        self.pages = sum(used) + spare + (len(lens) * max_pages if max_pages else 0)
        order = torch.randperm(self.pages, generator=g).tolist()
        self.table = torch.full((len(lens), self.max_pages), -1, dtype=torch.int32)
        for i, n in enumerate(used):
            for j in range(n):
                self.table[i, j] = order.pop()
        n, m = self.pages * heads * page * dim // 2, self.pages * heads * page * self.runs * 4
        self.guards = {"k": Guarded(n), "v": Guarded(n), "k_scales": Guarded(m), "v_scales": Guarded(m)}
        self.k = self.guards["k"].view(torch.int32, (self.pages, heads, page, dim // 8))
        self.v = self.guards["v"].view(torch.int32, (self.pages, heads, page // 16, dim, 2))
        self.k_scales = self.guards["k_scales"].view(torch.float16, (self.pages, heads, page, self.runs, 2))
        self.v_scales = self.guards["v_scales"].view(torch.float16, (self.pages, heads, page // 16, self.runs, 2, 16))
        for pool in (self.k, self.v):
            pool.copy_(torch.randint(-(1 << 31), 1 << 31, pool.shape, generator=g).to(torch.int32))
        filled = [max(n, 0) for n in lens] if filled is None else filled
        for scales, at in ((self.k_scales, 4), (self.v_scales, 4)):
            plain = scales.shape[:4] + scales.shape[5:]
            s = (torch.rand(plain, generator=g) * 0.2 + 0.1).half()
            o = (torch.randn(plain, generator=g) * 0.3 - 23.5 * s.float()).half()
            scales.copy_(torch.stack([s, o], dim=at).cuda())
        keep = torch.zeros(self.pages, page, dtype=torch.bool)          # places of tokens
        for i, n in enumerate(filled):
            for t in range(min(n, self.max_pages * page)):
                keep[int(self.table[i, t // page]), t % page] = True
        keep = keep.cuda()
        self.k_scales.masked_fill_(~keep[:, None, :, None, None], float("nan"))
        self.v_scales.masked_fill_(~keep.view(self.pages, 1, page // 16, 1, 1, 16), float("nan"))
        self.table_dev = self.table.cuda()
        self.lens_dev = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def remap(self, table):
        """The same pools under another table; what the sequences hold goes with them."""
        table = table.to(torch.int32)
        old = self.snapshot()
        for i, n in enumerate(self.lens):
            for j in range(-(-max(n, 0) // self.page)):
                a, b = int(self.table[i, j]), int(table[i, j])
                for x, y in ((self.k, old[0]), (self.k_scales, old[1]), (self.v, old[2]), (self.v_scales, old[3])):
                    x[b].copy_(y[a])
        self.table = table
        self.table_dev = table.cuda()

    def page_of(self, i, t):
        p = int(self.table[i, t // self.page]) if 0 <= t < self.max_pages * self.page else -1
        return p if 0 <= p < self.pages else None

    def raw(self, i, t, values):
        """codes [heads][dim], scales and offsets [heads][runs]"""
        p, s = self.page_of(i, t), t % self.page
        if values:
            return (unpack(self.v[p, :, s // 16, :, s % 16 // 8])[..., s % 8], self.v_scales[p, :, s // 16, :, 0, s % 16], self.v_scales[p, :, s // 16, :, 1, s % 16])
        return unpack(self.k[p, :, s]).flatten(-2), self.k_scales[p, :, s, :, 0], self.k_scales[p, :, s, :, 1]

    def wide(self, x):
        return x.repeat_interleave(self.block, dim=-1)[..., :self.dim]

    def read(self, i, t, values):
        """[heads][dim] in 64 bits, or None where there is no page."""
        if self.page_of(i, t) is None:
            return None
        code, s, o = self.raw(i, t, values)
        return ((code.double() + 16) * self.wide(s.double()) + self.wide(o.double())).half().double()

    def sequence(self, i, lo, hi):
        """keys and values [hi - lo][heads][dim] of a sequence in 64 bits, and which of them have a page"""
        t = torch.arange(lo, max(lo, hi))
        page = torch.where(t < self.max_pages * self.page, self.table[i, (t // self.page).clamp(max=self.max_pages - 1)].long(), -1)
        seen = ((page >= 0) & (page < self.pages)).cuda()
        p, s = page.clamp(0, self.pages - 1).cuda(), (t % self.page).cuda()
        k = (unpack(self.k[p, :, s]).flatten(-2).double() + 16) * self.wide(self.k_scales[p, :, s, :, 0].double()) + self.wide(self.k_scales[p, :, s, :, 1].double())
        code = torch.gather(unpack(self.v[p, :, s // 16, :, s % 16 // 8]), -1, (s % 8)[:, None, None, None].expand(len(t), self.heads, self.dim, 1))[..., 0]
        v = (code.double() + 16) * self.wide(self.v_scales[p, :, s // 16, :, 0, s % 16].double()) + self.wide(self.v_scales[p, :, s // 16, :, 1, s % 16].double())
        return k.half().double(), v.half().double(), seen

    def snapshot(self):
        return tuple(x.clone() for x in (self.k, self.k_scales, self.v, self.v_scales))

    def copy_of(self, before, values):
        return (before[2].clone(), before[3].clone()) if values else (before[0].clone(), before[1].clone())

    def accept(self, pool, scales, i, t, values):
        """Puts a token's codes, scales and offsets as they are now into a copy of the pools."""
        p, s = self.page_of(i, t), t % self.page
        if not values:
            pool[p, :, s] = self.k[p, :, s]
            scales[p, :, s] = self.k_scales[p, :, s]
            return
        at = (p, slice(None), s // 16, slice(None), s % 16 // 8)
        codes = unpack(pool[at])
        codes[..., s % 8] = unpack(self.v[at])[..., s % 8]
        pool[at] = pack(codes)
        scales[p, :, s // 16, :, :, s % 16] = self.v_scales[p, :, s // 16, :, :, s % 16]

    def same(self, pool, scales, values):
        mine, mine_s = (self.v, self.v_scales) if values else (self.k, self.k_scales)
        return torch.equal(pool, mine) and torch.equal(scales.view(torch.int16), mine_s.view(torch.int16))

    def struct(self):
        return cg.KvCache.make(self.k, self.v, self.k_scales, self.v_scales, self.table_dev, self.lens_dev, kv_heads=self.heads, head_dim=self.dim,
                               num_pages=self.pages, page_size=self.page, dtype=self.dtype, scale_block=self.block, num_seqs=len(self.lens),
                               max_pages=self.max_pages)

    def intact(self):
        torch.cuda.synchronize()
        return all(g.intact() for g in self.guards.values())

"""Paged caches, prompts and their definitions in 64 bits for the tests of codegemm_kv_append, codegemm_kv_gather, codegemm_attn_decode and
codegemm_attn_prompt.  Works from the documented layouts, element by element; shares no code with the library."""
from __future__ import annotations

import math

import torch

import paper_2512_17970_amd as cg
from gpu_util import Guarded, stream

QMAX = {cg.binding.KV_INT8: 127.0, cg.binding.KV_FP8: 448.0}


def rope_table(positions, rotary, base=10000.0):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / max(rotary, 1))
    return torch.stack([angle.cos(), angle.sin()], -1).float().cuda().contiguous()


class Cache:
    """A paged cache between canary bands; every place that holds no token holds `fill` (NaN where the type has one)."""

    def __init__(self, lens, *, heads=2, dim=64, page=16, dtype=cg.binding.KV_FP16, block=1, seed=0, spare=3, max_pages=None, scale=0.02, filled=None):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.heads, self.dim, self.page, self.dtype, self.block = list(lens), heads, dim, page, dtype, block
        used = [-(-max(n, 0) // page) for n in lens]
        self.max_pages = max_pages or max(1, max(used))
        self.pages = sum(used) + spare
        order = torch.randperm(self.pages, generator=g).tolist()
        self.table = torch.full((len(lens), self.max_pages), -1, dtype=torch.int32)
        for i, n in enumerate(used):
            for j in range(n):
                self.table[i, j] = order.pop()
        size = 2 if dtype == cg.binding.KV_FP16 else 1
        n = self.pages * heads * page * dim
        self.guards = {"k": Guarded(n * size), "v": Guarded(n * size)}
        self.blocks = page // block
        if size == 1:
            self.guards |= {"k_scales": Guarded(self.pages * heads * self.blocks * 4), "v_scales": Guarded(self.pages * heads * self.blocks * 4)}
        kind = torch.float16 if size == 2 else torch.uint8
        self.k = self.guards["k"].view(kind, (self.pages, heads, page, dim))
        self.v = self.guards["v"].view(kind, (self.pages, heads, page // 16, dim, 16))
        self.k_scales = self.guards["k_scales"].view(torch.float32, (self.pages, heads, self.blocks)) if size == 1 else None
        self.v_scales = self.guards["v_scales"].view(torch.float32, (self.pages, heads, self.blocks)) if size == 1 else None
        for pool, scales in ((self.k, self.k_scales), (self.v, self.v_scales)):
            pool.fill_(float("nan") if size == 2 else 0x7F if dtype == cg.binding.KV_FP8 else 0x55)      # 0x7F: a NaN in e4m3
            if scales is not None:
                scales.fill_(float("nan"))
        for i, n in enumerate(lens):                              # what the sequences hold
            for t in range(max(n, 0) if filled is None else filled[i]):
                for pool, scales, values in ((self.k, self.k_scales, False), (self.v, self.v_scales, True)):
                    if size == 2:
                        x = torch.randn(heads, dim, generator=g).half()
                    elif dtype == cg.binding.KV_INT8:
                        x = torch.randint(-127, 128, (heads, dim), generator=g).to(torch.int8).view(torch.uint8)
                    else:
                        x = torch.randint(0, 127, (heads, dim), generator=g).to(torch.uint8) + 128 * torch.randint(0, 2, (heads, dim), generator=g).to(torch.uint8)
                    self.place(pool, i, t, values).copy_(x.cuda())
                    if scales is not None and t % block == 0:
                        self.scale_of(scales, i, t).copy_(((torch.rand(heads, generator=g) + 0.5) * scale * (127 / QMAX[dtype])).cuda())
        self.table_dev = self.table.cuda()
        self.lens_dev = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def page_of(self, i, t):
        p = int(self.table[i, t // self.page]) if 0 <= t < self.max_pages * self.page else -1
        return p if 0 <= p < self.pages else None

    def place(self, pool, i, t, values):
        p, s = self.page_of(i, t), t % self.page
        return pool[p, :, s // 16, :, s % 16] if values else pool[p, :, s]

    def scale_of(self, scales, i, t):
        return scales[self.page_of(i, t), :, t % self.page // self.block]

    def value(self, codes):
        if self.dtype == cg.binding.KV_INT8:
            return codes.view(torch.int8).double()
        return codes.view(torch.float8_e4m3fn).double() if self.dtype == cg.binding.KV_FP8 else codes.double()

    def read(self, i, t, values):
        """[heads][dim] in 64 bits, or None where there is no page."""
        if self.page_of(i, t) is None:
            return None
        x = self.value(self.place(self.v if values else self.k, i, t, values).contiguous())
        scales = self.v_scales if values else self.k_scales
        return x if scales is None else x * self.scale_of(scales, i, t).double()[:, None]

    def struct(self):
        return cg.KvCache.make(self.k, self.v, self.k_scales, self.v_scales, self.table_dev, self.lens_dev, kv_heads=self.heads, head_dim=self.dim,
                               num_pages=self.pages, page_size=self.page, dtype=self.dtype, scale_block=self.block, num_seqs=len(self.lens),
                               max_pages=self.max_pages)

    def intact(self):
        torch.cuda.synchronize()
        return all(g.intact() for g in self.guards.values())


def attention(q, k, v, seen, scale):
    """q [heads][D], k, v [n][kv heads][D], seen [n]: one query in 64 bits, and per head a bound on the kernels' error:
    scores carry (D + 4) 2^-24 of the sum of their products' sizes, a weight that much of its size and the fp16 rounding (2^-11, or 2^-25 of
    the largest weight where it is a subnormal), the result its own rounding; sums in 32 bits add (n + 64) 2^-24 of the sizes."""
    Hq, D = q.shape
    r = Hq // k.shape[1]
    out, bound = torch.zeros(Hq, D, dtype=torch.float64, device=q.device), torch.zeros(Hq, D, dtype=torch.float64, device=q.device)
    if not bool(seen.any()):
        return out, bound
    k, v, q = k[seen], v[seen], q.double()
    n = k.shape[0]
    for h in range(Hq):
        kh, vh = k[:, h // r], v[:, h // r]
        s = (kh * q[h]).sum(-1) * scale
        p = torch.softmax(s, 0)
        out[h] = (p[:, None] * vh).sum(0)
        size = ((kh * q[h]).abs().sum(-1) * abs(scale)).max()
        each = 2.0 ** -11 + (2 * (D + 4) * 2.0 ** -24) * size + (n + 64) * 2.0 ** -24
        bound[h] = 1.01 * each * (p[:, None] * vh.abs()).sum(0) + 2.0 ** -11 * out[h].abs() + n * 2.0 ** -25 * vh.abs().max() + 2.0 ** -25
    return out, bound


def check(got, want, bound, what):
    got = got.double()
    assert torch.equal(got.isfinite(), want.isfinite()), f"{what}: {int((got.isfinite() != want.isfinite()).sum())} places are finite in one and not in the other"
    fine = want.isfinite()
    over = ((got - want).abs() > bound) & fine
    assert not bool(over.any()), f"{what}: {int(over.sum())} of {got.numel()} over the bound, worst {float(((got - want).abs() / bound)[over].max()):.2f} times"


WORKSPACE = {}


def workspace(nbytes):
    """One workspace for all calls, as a program has, initialised once."""
    if WORKSPACE.get("bytes", 0) < nbytes:
        g = Guarded(nbytes)
        cg.codegemm_workspace_init(g.t, nbytes, stream())
        WORKSPACE.update(bytes=nbytes, guard=g)
    return WORKSPACE["guard"].t, WORKSPACE["bytes"]


def counters_are_clear():
    torch.cuda.synchronize()
    g = WORKSPACE["guard"]
    return g.intact() and int(g.t[:65536 + (2 << 20)].view(torch.int32).abs().sum()) == 0


def decode(cache, q, *, window=0, scale=None, max_kv=None, out=None, q_stride=0, out_stride=0):
    B, Hq, D = q.shape
    d = cg.AttnDesc.make(Hq, cache.heads, D, num_seqs=B, total_q=B, max_kv=max_kv or max(1, max(cache.lens)), scale=D ** -0.5 if scale is None else scale, window=window,
                         q_stride=q_stride, out_stride=out_stride)
    c = cache.struct()
    ws, n = workspace(cg.codegemm_attn_decode_workspace_bytes(c, d))
    g = Guarded(B * Hq * D * 2)
    mine = g.view(torch.float16, (B, Hq, D)).fill_(float("nan")) if out is None else out
    cg.codegemm_attn_decode(c, d, q, mine, ws, n, stream())
    assert g.intact() and cache.intact() and counters_are_clear()
    return mine


def decode_exact(cache, q, window=0, scale=None):
    out, bound = [], []
    for i, n in enumerate(cache.lens):
        lo = max(0, n - window) if window else 0
        held = [t for t in range(lo, n) if cache.page_of(i, t) is not None]
        if held:
            k = torch.stack([cache.read(i, t, False) for t in held])
            v = torch.stack([cache.read(i, t, True) for t in held])
        else:
            k = v = torch.zeros(0, cache.heads, cache.dim, dtype=torch.float64, device="cuda")
        o, b = attention(q[i], k, v, torch.ones(len(held), dtype=torch.bool, device="cuda"), cache.dim ** -0.5 if scale is None else scale)
        out.append(o)
        bound.append(b)
    return torch.stack(out), torch.stack(bound)


def starts(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def prompt(q, k, v, new, total, *, window=0, causal=True, scale=None, max_kv=None, strides=(0, 0, 0, 0), out=None):
    Hq, Hk, D = q.shape[1], k.shape[1], q.shape[2]
    d = cg.AttnDesc.make(Hq, Hk, D, num_seqs=len(new), total_q=sum(new), total_kv=sum(total), max_kv=max_kv or max(1, max(total)), scale=D ** -0.5 if scale is None else scale,
                         window=window, causal=causal, q_stride=strides[0], k_stride=strides[1], v_stride=strides[2], out_stride=strides[3])
    ws, n = workspace(cg.codegemm_attn_prompt_workspace_bytes(d))
    g = Guarded(sum(new) * Hq * D * 2)
    mine = g.view(torch.float16, (sum(new), Hq, D)).fill_(float("nan")) if out is None else out
    cu_kv = None if new == total else starts(total)
    cg.codegemm_attn_prompt(d, q, k, v, starts(new), cu_kv, mine, ws, n, stream())
    assert g.intact() and counters_are_clear()
    return mine


def prompt_exact(q, k, v, new, total, *, window=0, causal=True, scale=None, rows=None):
    """rows: of the packed queries, those that are wanted (all)."""
    out, bound, q0, k0 = [], [], 0, 0
    for n, t in zip(new, total):
        kd, vd, key = k[k0:k0 + t].double(), v[k0:k0 + t].double(), torch.arange(t, device="cuda")
        for j in range(n):
            if rows is not None and q0 + j not in rows:
                continue
            at = t - n + j
            seen = torch.ones(t, dtype=torch.bool, device="cuda")
            if causal:
                seen &= key <= at
            if window:
                seen &= key > at - window
            o, b = attention(q[q0 + j], kd, vd, seen, q.shape[2] ** -0.5 if scale is None else scale)
            out.append(o)
            bound.append(b)
        q0 += n
        k0 += t
    return torch.stack(out), torch.stack(bound)


def rotated(x, weight, positions, rope, rotary, interleaved, eps):
    """x [tokens][heads][D] in 64 bits: the norm and the rotation of every position."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    out = x.clone()
    for i in range(rotary // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
        at = positions.clamp(0, max(0, rope.shape[0] - 1))
        c, s = rope[at, i, 0].double()[:, None], rope[at, i, 1].double()[:, None]
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
    return out

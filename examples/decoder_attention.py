"""The attention part of a decoder block on codebook-quantised projections, as a server runs it:

    x -> q, k, v (codegemm_gemm, for single tokens codegemm_gemm_grouped) -> into the paged cache, rotated (codegemm_kv_append)
      -> attention: of prompts (codegemm_attn_prompt; of a prompt's further chunks over its cached prefix too, codegemm_kv_gather),
         of single tokens over the cache (codegemm_attn_decode) -> output projection (codegemm_gemm)

A step of single tokens is one HIP graph, in which the sequences' lengths grow on the device.  Its workspace stays where the graph finds it; that of
prompts grows with them.

    python examples/decoder_attention.py                    # 32 and 8 heads of 128, cache in int8: times and a check of the two paths
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2512_17970_amd as cg  # noqa: E402


def stream() -> int:
    return torch.cuda.current_stream().cuda_stream


class Linear:
    """A codebook-quantised layer with synthetic weights of variance 1 / K."""

    def __init__(self, K: int, N: int, gen, v: int = 8, m: int = 2):
        self.K, self.N, self.v, self.m = K, N, v, m
        self.codes = torch.randint(0, 256, (m, N, K // v), generator=gen, device="cuda", dtype=torch.uint8)
        self.codebooks = torch.randn(m, 256, v, generator=gen, device="cuda").half()
        self.scales = ((0.75 + 0.5 * torch.rand(N, generator=gen, device="cuda")) * (K * m) ** -0.5).half()
        desc = self.desc(1)
        self.packed = torch.empty(cg.codegemm_packed_codes_bytes(desc), dtype=torch.uint8, device="cuda")
        cg.codegemm_pack_codes(desc, None, self.codes, self.packed, stream())

    def desc(self, rows: int) -> cg.Desc:
        return cg.Desc.make(rows, self.K, self.N, self.v, self.m)

    def member(self, y):
        return self.N, self.packed, self.codebooks, self.scales, y

    def __call__(self, x, y, workspace) -> None:
        cg.codegemm_gemm(self.desc(x.shape[0]), None, x, self.packed, self.codebooks, self.scales, y, workspace, workspace.numel(), stream())


class DecoderAttention:
    def __init__(self, hidden: int, q_heads: int, kv_heads: int, head_dim: int, *, num_seqs: int, max_tokens: int,
                 kv_dtype: int = cg.KV_INT8, page_size: int = 64, scale_block: int = 16, theta: float = 500000.0, seed: int = 1):
        """max_tokens: of a sequence."""
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.hidden, self.q_heads, self.kv_heads, self.head_dim, self.num_seqs, self.max_tokens = hidden, q_heads, kv_heads, head_dim, num_seqs, max_tokens
        self.q, self.k, self.v = (Linear(hidden, heads * head_dim, gen) for heads in (q_heads, kv_heads, kv_heads))
        self.o = Linear(q_heads * head_dim, hidden, gen)
        freq = theta ** (-torch.arange(0, head_dim, 2, dtype=torch.float64, device="cuda") / head_dim)
        angle = torch.arange(max_tokens, dtype=torch.float64, device="cuda")[:, None] * freq
        self.rope = torch.stack([angle.cos(), angle.sin()], dim=-1).float().contiguous()

        # The cache: every sequence has its pages from the start, in random order; a server would hand them out as sequences grow.
        max_pages = -(-max_tokens // page_size)
        pages = num_seqs * max_pages
        self.table = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32).view(num_seqs, max_pages).contiguous()
        self.lens = torch.zeros(num_seqs, dtype=torch.int32, device="cuda")
        self.held = [0] * num_seqs                                       # the same on the host
        layout = dict(kv_heads=kv_heads, head_dim=head_dim, num_pages=pages, page_size=page_size, dtype=kv_dtype, scale_block=scale_block, num_seqs=num_seqs,
                      max_pages=max_pages)
        plain = cg.KvCache.make(None, None, None, None, None, None, **layout)
        pool = [torch.empty(cg.codegemm_kv_pool_bytes(plain), dtype=torch.uint8, device="cuda") for _ in range(2)]
        scale_bytes = cg.codegemm_kv_scales_bytes(plain)
        scales = [torch.empty(scale_bytes // 4, device="cuda") if scale_bytes else None for _ in range(2)]
        self.kept = pool, scales
        self.cache = cg.KvCache.make(*pool, *scales, self.table, self.lens, **layout)

        self.step_attn = cg.AttnDesc.make(q_heads, kv_heads, head_dim, num_seqs=num_seqs, total_q=num_seqs, max_kv=max_tokens, scale=head_dim ** -0.5)
        self.step_group = cg.Desc.make(num_seqs, hidden, self.q.N + 2 * self.k.N, self.q.v, self.q.m)
        need = [cg.codegemm_attn_decode_workspace_bytes(self.cache, self.step_attn)] + [cg.codegemm_workspace_bytes(layer.desc(num_seqs)) for layer in (self.q, self.k, self.o)]
        if num_seqs <= 32:
            need.append(cg.codegemm_grouped_workspace_bytes(self.step_group, None, [self.q.N, self.k.N, self.v.N]))
        self.step_workspace, self.workspace = self.new_workspace(max(need)), None

    @staticmethod
    def new_workspace(nbytes: int) -> torch.Tensor:
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        cg.codegemm_workspace_init(ws, nbytes, stream())
        return ws

    def buffers(self, tokens: int):
        half = lambda *shape: torch.empty(*shape, dtype=torch.float16, device="cuda")  # noqa: E731
        heads = [half(tokens, n, self.head_dim) for n in (self.q_heads, self.kv_heads, self.kv_heads, self.q_heads)]
        return (*heads, half(tokens, self.hidden))

    def append(self, cu, q, k, v) -> None:
        desc = cg.AppendDesc.make(q.shape[0], self.q_heads, rotary_dim=self.head_dim, rope_positions=self.max_tokens)
        cg.codegemm_kv_append(self.cache, desc, cu, q, k, v, None, None, self.rope, q, k, stream())      # q and k turn in place

    def prompts(self, x, new) -> torch.Tensor:
        """x [sum(new)][hidden]: the next new[i] tokens of sequence i, after those that it holds."""
        starts = lambda n: torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device="cuda")  # noqa: E731
        tokens, past = sum(new), list(self.held)
        assert len(new) == self.num_seqs and x.shape == (tokens, self.hidden) and all(p + n <= self.max_tokens for p, n in zip(past, new))
        self.held = [p + n for p, n in zip(past, new)]
        self.lens += torch.tensor(new, dtype=torch.int32, device="cuda")
        q, k, v, heads, y = self.buffers(tokens)
        total = sum(self.held) if any(past) else tokens
        attn = cg.AttnDesc.make(self.q_heads, self.kv_heads, self.head_dim, num_seqs=self.num_seqs, total_q=tokens, total_kv=total, max_kv=max(self.held),
                                scale=self.head_dim ** -0.5, causal=True)
        need = max(cg.codegemm_attn_prompt_workspace_bytes(attn), *(cg.codegemm_workspace_bytes(layer.desc(tokens)) for layer in (self.q, self.k, self.o)))
        if self.workspace is None or self.workspace.numel() < need:
            self.workspace = self.new_workspace(need)
        for layer, to in ((self.q, q), (self.k, k), (self.v, v)):
            layer(x, to, self.workspace)
        cu, cu_kv = starts(new), None
        self.append(cu, q, k, v)
        if any(past):                                                    # prefixes in the cache: all keys come from there
            cu_kv = starts(self.held)
            k, v = (torch.empty(total, self.kv_heads, self.head_dim, dtype=torch.float16, device="cuda") for _ in range(2))
            cg.codegemm_kv_gather(self.cache, total, cu_kv, None, k, v, stream())
        cg.codegemm_attn_prompt(attn, q, k, v, cu, cu_kv, heads, self.workspace, self.workspace.numel(), stream())
        self.o(heads.view(tokens, -1), y, self.workspace)
        return y

    def step(self, x, buffers) -> torch.Tensor:
        """x [num_seqs][hidden]: one token more per sequence.  Allocates nothing and does not look at the lengths, so a graph can hold it."""
        q, k, v, heads, y = buffers
        self.lens += 1
        if self.num_seqs <= 32:
            members = [layer.member(to) for layer, to in ((self.q, q), (self.k, k), (self.v, v))]
            cg.codegemm_gemm_grouped(self.step_group, None, x, members, self.step_workspace, self.step_workspace.numel(), stream())
        else:
            for layer, to in ((self.q, q), (self.k, k), (self.v, v)):
                layer(x, to, self.step_workspace)
        self.append(None, q, k, v)
        cg.codegemm_attn_decode(self.cache, self.step_attn, q, heads, self.step_workspace, self.step_workspace.numel(), stream())
        self.o(heads.view(self.num_seqs, -1), y, self.step_workspace)
        return y

    def capture(self, x, buffers) -> torch.cuda.CUDAGraph:
        """A step as a graph; run step() once before.  Capturing runs nothing, and every replay is a step (the caller counts `held`)."""
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            self.step(x, buffers)
        torch.cuda.current_stream().wait_stream(side)
        return graph


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--q-heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--kv", choices=("fp16", "int8", "fp8"), default="int8")
    ap.add_argument("--seqs", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=1000, help="tokens of the longest prompt")
    ap.add_argument("--steps", type=int, default=64)
    a = ap.parse_args()
    kv = {"fp16": cg.KV_FP16, "int8": cg.KV_INT8, "fp8": cg.KV_FP8}[a.kv]
    new = [max(1, a.prompt * (i + 1) // a.seqs) for i in range(a.seqs)]
    block = DecoderAttention(a.hidden, a.q_heads, a.kv_heads, a.head_dim, num_seqs=a.seqs, max_tokens=2 * a.prompt + a.steps + 2, kv_dtype=kv)

    def timed(what, tokens, run):
        torch.cuda.synchronize()
        t = time.perf_counter()
        out = run()
        torch.cuda.synchronize()
        t = time.perf_counter() - t
        print(f"{what:34s} {t * 1e6:10.1f} us  {tokens / t:12.0f} tokens/s", flush=True)
        return out

    x = torch.randn(sum(new), a.hidden, device="cuda").half()
    block.prompts(x, new)
    block.lens.zero_()
    block.held = [0] * a.seqs
    timed(f"prompts of {new[0]} .. {new[-1]}", sum(new), lambda: block.prompts(x, new))
    timed("as many tokens behind them", sum(new), lambda: block.prompts(x, new))
    token, buffers = torch.randn(a.seqs, a.hidden, device="cuda").half(), block.buffers(a.seqs)
    block.step(token, buffers)
    graph = block.capture(token, buffers)

    def steps():
        for _ in range(a.steps):
            graph.replay()
    timed(f"{a.steps} steps, cache of {sum(block.held)} tokens", a.steps * a.seqs, steps)

    # One token more, by the cache and as a chunk of one: the same but for roundings.
    lens = block.lens.clone()
    one = block.step(token, buffers).double()
    block.lens.copy_(lens)
    block.held = lens.tolist()
    other = block.prompts(token, [1] * a.seqs).double()
    error = float((one - other).norm() / other.norm())
    print(f"a step against a chunk of one token: relative error {error:.1e}")
    assert error < 2.0 ** -7


if __name__ == "__main__":
    main()

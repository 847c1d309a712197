"""examples/decoder_attention.py: prompts, chunks and single tokens through quantised projections, the cache and attention, against the same in 64
bits from the dequantised weights."""
import importlib.util
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
import paper_2512_17970_amd as cg  # noqa: E402

pytestmark = pytest.mark.gpu

AT = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_attention.py")
spec = importlib.util.spec_from_file_location("decoder_attention", AT)
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)

# Relative error of a token's result.  Roundings to fp16 (2^-11): of q, k, v by the projection and k, q by the rotation, the weights, the result; scores
# of up to 8 in size turn those of q and k into 4 x 8 x 2^-11 of a weight at worst, so 2^-6 of the result; the cache's 8 bits add half a step,
# 1/254 (int8) or 2^-4 (fp8) of the largest of a block's values at worst and a third of it on average, to values and, through the scores, to weights.
BOUND = {cg.KV_FP16: 2.0 ** -6, cg.KV_INT8: 2.0 ** -4, cg.KV_FP8: 2.0 ** -2}


def dense(layer):
    w = sum(layer.codebooks[c][layer.codes[c].long()].double() for c in range(layer.m)).reshape(layer.N, layer.K)
    return w * layer.scales.double()[:, None]


class Exact:
    """The block in 64 bits, every sequence by itself."""

    def __init__(self, block):
        self.b, self.w = block, {n: dense(getattr(block, n)) for n in "qkvo"}
        self.keys, self.values = ([torch.zeros(0, block.kv_heads, block.head_dim, dtype=torch.float64, device="cuda") for _ in range(block.num_seqs)] for _ in range(2))

    def turn(self, x, first):
        rope = self.b.rope[first:first + x.shape[0]].double()
        c, s, half = rope[:, None, :, 0], rope[:, None, :, 1], self.b.head_dim // 2
        return torch.cat([x[..., :half] * c - x[..., half:] * s, x[..., half:] * c + x[..., :half] * s], dim=-1)

    def more(self, x, new):
        out, at = [], 0
        for i, n in enumerate(new):
            rows, past = x[at:at + n].double(), self.keys[i].shape[0]
            at += n
            q, k, v = ((rows @ self.w[c].T).view(n, -1, self.b.head_dim) for c in "qkv")
            self.keys[i] = torch.cat([self.keys[i], self.turn(k, past)])
            self.values[i] = torch.cat([self.values[i], v])
            r = self.b.q_heads // self.b.kv_heads
            keys, values = (t[i].repeat_interleave(r, dim=1).transpose(0, 1) for t in (self.keys, self.values))
            scores = (self.turn(q, past).transpose(0, 1) * self.b.head_dim ** -0.5) @ keys.transpose(1, 2).contiguous()
            ahead = torch.arange(past + n, device="cuda")[None, :] > past + torch.arange(n, device="cuda")[:, None]
            p = torch.softmax(scores.masked_fill(ahead, float("-inf")), dim=-1)
            out.append((p @ values).transpose(0, 1).reshape(n, -1) @ self.w["o"].T)
        return torch.cat(out)


def close(got, want, bound, what):
    error = (got.double() - want).norm(dim=-1) / want.norm(dim=-1)
    assert bool((error < bound).all()), f"{what}: {float(error.max()):.2e}"


@pytest.mark.parametrize("kv", [cg.KV_FP16, cg.KV_INT8, cg.KV_FP8])
@pytest.mark.parametrize("hidden,q_heads,kv_heads,head_dim,seqs", [(512, 8, 2, 64, 4), (1024, 8, 8, 128, 1), (256, 4, 1, 128, 35)])
def test_block(kv, hidden, q_heads, kv_heads, head_dim, seqs):
    new = [(37 * i) % 90 + 1 for i in range(seqs)]
    block = example.DecoderAttention(hidden, q_heads, kv_heads, head_dim, num_seqs=seqs, max_tokens=300, kv_dtype=kv, page_size=32, scale_block=8)
    exact, gen = Exact(block), torch.Generator(device="cuda").manual_seed(3)
    tokens = lambda n: torch.randn(n, hidden, generator=gen, device="cuda").half()  # noqa: E731
    x = tokens(sum(new))
    close(block.prompts(x, new), exact.more(x, new), BOUND[kv], "prompts")
    more = [(11 * i) % 40 for i in range(seqs)]
    more[0] = 50
    x = tokens(sum(more))
    close(block.prompts(x, more), exact.more(x, more), BOUND[kv], "chunks")
    token, buffers = tokens(seqs), block.buffers(seqs)
    close(block.step(token, buffers), exact.more(token, [1] * seqs), BOUND[kv], "step")
    graph = block.capture(token, buffers)
    for k in range(5):
        token.copy_(tokens(seqs))
        graph.replay()
        torch.cuda.synchronize()
        close(buffers[-1], exact.more(token, [1] * seqs), BOUND[kv], f"replay {k}")


def test_command():
    out = subprocess.run([sys.executable, AT, "--hidden", "512", "--q-heads", "8", "--kv-heads", "2", "--head-dim", "64", "--prompt", "100", "--steps", "3", "--seqs", "3"],
                         capture_output=True, text=True, timeout=100)
    assert out.returncode == 0 and "relative error" in out.stdout, out.stderr[-2000:]

"""A cache with a budget, as a server runs it: prompts, chunks and captured steps that keep count of what their tokens attend to, evictions between them, and appends
behind these (examples/decoder_attention.py), in every type of cache; against the same in 64 bits, which loses the same tokens."""
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
import paper_2512_17970_amd as cg  # noqa: E402
from test_gpu_decoder_attention import AT, BOUND, Exact, close, example  # noqa: E402

pytestmark = pytest.mark.gpu

# 4 bits: a code is off by up to 1/30 of its run's range, which is some 4 standard deviations of 32 values, so by 0.08 of one on average: as much in values, and, as
# the scores have a standard deviation of about 1, in weights; 0.12 together, and twice that is the bound.
BOUNDS = dict(BOUND) | {cg.KV_INT4: 2.0 ** -2}


class Budgeted(Exact):
    """keys, values: [kv head] of every sequence has tokens of its own; weights: what each of them has got so far."""

    def __init__(self, block):
        super().__init__(block)
        self.at = [0] * block.num_seqs                  # tokens so far, with those that are gone
        self.weights = [torch.zeros(block.kv_heads, 0, dtype=torch.float64, device="cuda") for _ in range(block.num_seqs)]

    def more(self, x, new):
        out, row, b = [], 0, self.b
        for i, n in enumerate(new):
            rows, past = x[row:row + n].double(), self.keys[i].shape[0]
            row += n
            q, k, v = ((rows @ self.w[c].T).view(n, -1, b.head_dim) for c in "qkv")
            self.keys[i] = torch.cat([self.keys[i], self.turn(k, self.at[i])])
            self.values[i] = torch.cat([self.values[i], v])
            r = b.q_heads // b.kv_heads
            keys, values = (t[i].repeat_interleave(r, dim=1).transpose(0, 1) for t in (self.keys, self.values))
            scores = (self.turn(q, self.at[i]).transpose(0, 1) * b.head_dim ** -0.5) @ keys.transpose(1, 2).contiguous()
            self.at[i] += n
            ahead = torch.arange(past + n, device="cuda")[None, :] > past + torch.arange(n, device="cuda")[:, None]
            p = torch.softmax(scores.masked_fill(ahead, float("-inf")), dim=-1)
            had = torch.cat([self.weights[i], torch.zeros(b.kv_heads, n, dtype=torch.float64, device="cuda")], dim=1)
            self.weights[i] = had + p[:, max(0, n - b.observers):].reshape(b.kv_heads, -1, past + n).sum(1)
            out.append((p @ values).transpose(0, 1).reshape(n, -1) @ self.w["o"].T)
        return torch.cat(out)

    def evict(self, i, stay):
        """stay [kv head][n]: positions"""
        at = stay.T[..., None].expand(-1, -1, self.b.head_dim)
        self.keys[i], self.values[i] = (t[i].gather(0, at) for t in (self.keys, self.values))
        self.weights[i] = self.weights[i].gather(1, stay)


def weights_of(block, i):
    n, page = int(block.lens[i]), block.scores.shape[2]
    t = torch.arange(n, device="cuda")
    return block.scores[block.table[i].long()[t // page], :, t % page].T


def evict(block, exact, bound):
    """One eviction of both, by the scores that the device has, which are near those in 64 bits."""
    lens, shift, first, last = block.lens.tolist(), block.shift.tolist(), block.evict_desc.keep_first, block.evict_desc.keep_last
    assert lens == [k.shape[0] for k in exact.keys]
    left = []
    for i, n in enumerate(lens):
        got = weights_of(block, i)
        assert float((got.double() - exact.weights[i]).norm()) <= bound * float(exact.weights[i].norm())
        rank = got.clone()
        rank[:, :first], rank[:, max(0, n - last):] = float("inf"), float("inf")
        stay = torch.sort(torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :block.budget], dim=1).values
        exact.evict(i, stay)
        left.append(got.gather(1, stay))
    block.held = lens
    block.evict()
    torch.cuda.synchronize()
    assert block.lens.tolist() == [min(n, block.budget) for n in lens] == block.held
    assert block.shift.tolist() == [s + max(0, n - block.budget) for s, n in zip(shift, lens)] == block.gone
    both = torch.cat([block.table, block.spare], dim=1).flatten().tolist()
    assert sorted(both) == list(range(len(both)))       # no page is lost
    for i, want in enumerate(left):
        assert torch.equal(weights_of(block, i), want)


@pytest.mark.parametrize("kv", [cg.KV_FP16, cg.KV_INT8, cg.KV_FP8, cg.KV_INT4])
@pytest.mark.parametrize("hidden,q_heads,kv_heads,head_dim,seqs,page", [(512, 8, 2, 64, 4, 32), (1024, 8, 8, 128, 1, 64), (256, 4, 1, 128, 35, 16)])
def test_block_with_a_budget(kv, hidden, q_heads, kv_heads, head_dim, seqs, page):
    new = [(37 * i) % 90 + 61 for i in range(seqs)]
    block = example.DecoderAttention(hidden, q_heads, kv_heads, head_dim, num_seqs=seqs, max_tokens=300, kv_dtype=kv, page_size=page,
                                     scale_block=32 if kv == cg.KV_INT4 else 8, budget=80, keep_first=2, keep_last=10, observers=16)
    exact, gen, bound = Budgeted(block), torch.Generator(device="cuda").manual_seed(3), BOUNDS[kv]
    tokens = lambda n: torch.randn(n, hidden, generator=gen, device="cuda").half()  # noqa: E731
    x = tokens(sum(new))
    close(block.prompts(x, new), exact.more(x, new), bound, "prompts")
    evict(block, exact, bound)
    more = [(11 * i) % 40 for i in range(seqs)]
    more[0] = 50
    x = tokens(sum(more))
    close(block.prompts(x, more), exact.more(x, more), bound, "chunks")
    evict(block, exact, bound)
    token, buffers = tokens(seqs), block.buffers(seqs)
    close(block.step(token, buffers), exact.more(token, [1] * seqs), bound, "step")
    graph = block.capture(token, buffers)
    for k in range(9):
        token.copy_(tokens(seqs))
        graph.replay()
        torch.cuda.synchronize()
        close(buffers[-1], exact.more(token, [1] * seqs), bound, f"replay {k}")
        if k % 3 == 2:
            evict(block, exact, bound)


def test_command():
    out = subprocess.run([sys.executable, AT, "--hidden", "512", "--q-heads", "8", "--kv-heads", "2", "--head-dim", "64", "--prompt", "100", "--steps", "3", "--seqs", "3",
                          "--kv", "int4", "--budget", "50"], capture_output=True, text=True, timeout=100)
    assert out.returncode == 0 and "eviction" in out.stdout and "relative error" in out.stdout, out.stderr[-2000:]

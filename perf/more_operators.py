"""What keeps a long context in less memory, as cases that can be timed and checked: a cache in 4 bits, and tokens that leave a cache.

A case is a pass through one of the operators:
  append   the new tokens' queries and keys are normalised per head (where the model has such norms) and rotated, keys and values go into a
           cache in 4 bits, and what it then holds for them is read back in fp16, as a prompt that is worked off in chunks does;
  decode   attention of one token per sequence over its cache in 4 bits;
  scores   the softmax weights that every cached token gets, summed over queries and over the heads that share its key: of the single tokens of a
           step, beside the attention itself, or of the last queries of prompts;
  evict    of every sequence and key head the tokens with the highest sums, with the first and the last ones, go to pages of their own; 8 and 4
           bits are read back in fp16, as the prompt's next chunk needs them.
Heads are those of the repository's decoder blocks (8B: 32 query and 8 key heads, 70B: 64 and 8, of 128) and of layers between them.
With `own` false, run() is elementary torch in 32 bits; exact() is the definition in 64 bits, sequence by sequence.
"""
from __future__ import annotations

import math
import random

import torch

own = False

KV_TYPES = {"fp16": 0, "int8": 1, "fp8": 2, "int4": 4}         # how the cache holds a value
QMAX = {"int8": 127.0, "fp8": 448.0}
WORKSPACE = 64 << 20                                           # of the program, for all its layers


def _append(name, q_heads, kv_heads, head_dim, block, page, seqs, new, past, mix, rotary=None, interleaved=False, norm=False):
    return {"name": name, "op": "append", "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "kv": "int4", "block": block, "page": page,
            "seqs": seqs, "new": new, "past": past, "mix": mix, "rotary": head_dim if rotary is None else rotary, "interleaved": interleaved, "norm": norm}


def _decode(name, q_heads, kv_heads, head_dim, block, page, seqs, longest, mix, window=0):
    return {"name": name, "op": "decode", "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "kv": "int4", "block": block, "page": page,
            "seqs": seqs, "longest": longest, "mix": mix, "window": window}


def _scores(name, q_heads, kv_heads, head_dim, kv, block, page, seqs, longest, queries, mix, window=0):
    """queries: of each sequence; 1: with the attention of these single tokens."""
    return {"name": name, "op": "scores", "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "kv": kv, "block": block, "page": page,
            "seqs": seqs, "longest": longest, "queries": queries, "mix": mix, "window": window}


def _evict(name, kv_heads, head_dim, kv, block, page, seqs, longest, budget, first, last, mix):
    return {"name": name, "op": "evict", "kv_heads": kv_heads, "head_dim": head_dim, "kv": kv, "block": block, "page": page, "seqs": seqs,
            "longest": longest, "budget": budget, "first": first, "last": last, "mix": mix}


def listed():
    return [
        # one token of one sequence of the 8B block: launch latency
        _append("append_8b_1_token", 32, 8, 128, 32, 64, 1, 1, 700, 0),
        # the prompts of five sequences, the largest batch of the repository's prompts four times over
        _append("append_70b_prompts", 64, 8, 128, 64, 64, 5, 1900, 0, 1),
        # one sequence of the 8B block: latency
        _decode("decode_8b_1_seq", 32, 8, 128, 32, 64, 1, 701, 2),
        # an ordinary step of the 70B block: 32 sequences of some thousand tokens
        _decode("decode_70b_32_seqs", 64, 8, 128, 32, 64, 32, 8192, 3),
        # three long documents, large pages
        _decode("decode_70b_long", 64, 8, 128, 64, 256, 3, 100001, 4),
        # every query head with its own keys, ragged, a window, a slot without a sequence
        _decode("decode_mha_window", 20, 20, 64, 32, 16, 13, 2222, 5, window=1500),
        # a step of one sequence that keeps count of what its tokens attend to: latency
        _scores("scores_8b_step", 32, 8, 128, "int4", 32, 64, 1, 701, 1, 6),
        # the same of 32 sequences of the 70B block
        _scores("scores_70b_step", 64, 8, 128, "int4", 32, 64, 32, 8192, 1, 7),
        # the last 32 queries of four prompts, which say what of them is to be kept, over 8 bits
        _scores("scores_70b_prompts", 64, 8, 128, "int8", 16, 64, 4, 8192, 32, 8),
        # one sequence of the 8B block back to its budget, fp16
        _evict("evict_8b_1_seq", 8, 128, "fp16", 1, 64, 1, 1111, 701, 4, 64, 9),
        # prompts to a quarter, 8 bits with blocks of 16 tokens
        _evict("evict_70b_prompts_int8", 8, 128, "int8", 16, 64, 5, 8192, 2048, 4, 128, 10),
        # the largest: three long documents to a third, 4 bits, large pages
        _evict("evict_70b_long", 8, 128, "int4", 64, 256, 3, 100001, 33333, 16, 1000, 11),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "scores", "scores", "evict", "evict"])
    kv_heads = rng.choice([1, 2, 4, 8])
    q_heads = kv_heads * rng.choice([1, 2, 4, 5, 7, 8])
    kv = "int4" if op in ("append", "decode") else rng.choice(["int4", "int4", "int8", "fp8", "fp16"])
    head_dim = rng.choice([64, 96, 128, 128, 128, 256] if kv == "int4" else [64, 80, 128, 128, 256])
    page = rng.choice([16, 32, 64, 128, 256])
    block = 1 if kv == "fp16" else rng.choice([32, 32, 64, 128]) if kv == "int4" else rng.choice([b for b in (1, 4, 16, 64) if b <= page])
    mix = rng.randrange(1 << 30)
    if op == "append":
        seqs = _log(rng, 1, 64)
        case = _append("", q_heads, kv_heads, head_dim, block, page, seqs, rng.choice([1, _log(rng, 1, 8192 // seqs)]), rng.choice([0, _log(rng, 1, 8192)]), mix,
                       rotary=rng.choice([head_dim, head_dim // 32 * 16, 0]), interleaved=rng.random() < 0.4, norm=rng.random() < 0.4)
    elif op == "decode":
        seqs = _log(rng, 1, 64)
        case = _decode("", q_heads, kv_heads, head_dim, block, page, seqs, _log(rng, 1, 200000 // seqs), mix, window=rng.choice([0, 0, _log(rng, 1, 4096)]))
    elif op == "scores":
        seqs, queries = _log(rng, 1, 32), rng.choice([1, 1, _log(rng, 2, 64)])
        longest = _log(rng, 1, min(100000, (200000 if queries == 1 else 1000000 // (queries * max(1, q_heads // 8))) // seqs))
        case = _scores("", q_heads, kv_heads, head_dim, kv, block, page, seqs, longest, queries, mix, window=rng.choice([0, 0, 0, _log(rng, 1, 4096)]))
    else:
        seqs = _log(rng, 1, 32)
        longest = _log(rng, 1, 100000 // seqs)
        budget = _log(rng, 1, longest)
        first = rng.choice([0, min(budget, 4)])
        case = _evict("", kv_heads, head_dim, kv, block, page, seqs, longest, budget, first, rng.choice([0, (budget - first) // rng.choice([1, 2, 8, 32])]), mix)
    del case["name"]
    return case


# ---- lengths: of the case alone, so that work() knows them ------------------------------------------------------------------

def _lengths(case):
    """(new tokens or queries, tokens in all) of every sequence."""
    rng, n = random.Random(case["mix"]), case["seqs"]
    if case["op"] != "append":
        total = [max(1, int(case["longest"] * (1 - rng.random() * 0.5))) for _ in range(n)]
        total[rng.randrange(n)] = case["longest"]
        if n > 4:
            total[n // 2] = 0                                          # a slot without a sequence
        single = case["op"] == "decode" or case.get("queries") == 1
        return [1 if single else min(case.get("queries", 0), t) for t in total], total
    new = [case["new"] if k == 0 else max(1, int(case["new"] * rng.random())) for k in range(n)]
    if case["new"] > 1 and case["past"] == 0:
        new = [max(1, int(case["new"] * (0.7 + 0.3 * rng.random()))) for _ in range(n)]
    past = [int(case["past"] * rng.random()) if case["past"] else 0 for _ in range(n)]
    return new, [a + b for a, b in zip(new, past)]


def _kept(case):
    return [min(t, case["budget"]) for t in _lengths(case)[1]]


def _starts(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


# ---- what a program has in hand -----------------------------------------------------------------------------------------------
# The cache in 4 bits.  Eight values are the 32-bit word in which value j has bits 4 (j / 2) + 16 (j % 2) .. + 3: of keys eight dimensions of a token,
# of values eight tokens of a dimension.  Value = fp16((code + 16) * scale + offset), scale and offset in fp16 for every token and `block` dimensions.

def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _runs(case):
    """Runs of dimensions with a scale of their own."""
    return -(-case["head_dim"] // case["block"])


def _rope_table(positions, rotary):
    """cos and sin of position * 500000^(-2i/R) as [positions][R/2][2]"""
    freq = 500000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / rotary)
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], dim=-1).float().contiguous()


def _pool_shapes(case, pages):
    """(shape of the pool, of its scales) for keys and for values"""
    H, D, page = case["kv_heads"], case["head_dim"], case["page"]
    if case["kv"] == "int4":
        G = _runs(case)
        return ((pages, H, page, D // 8), (pages, H, page, G, 2)), ((pages, H, page // 16, D, 2), (pages, H, page // 16, G, 2, 16))
    scales = (pages, H, page // case["block"])
    return ((pages, H, page, D), scales), ((pages, H, page // 16, D, 16), scales)


def _table(case, gen, total):
    """Pages in random order, one that no sequence has among them."""
    used = [-(-t // case["page"]) for t in total]
    most, pages = max(1, max(used)), sum(used) + 1
    order = torch.randperm(pages, generator=gen, device="cuda")
    starts = torch.tensor(_starts(used)[:-1], device="cuda")
    at = (starts[:, None] + torch.arange(most, device="cuda")).clamp(max=pages - 1)
    return {"pages": pages, "most": most, "table": order[at].to(torch.int32).contiguous(), "lens": _ints(total)}


def _cache(case, gen, total):
    """A pool of pages, codes and scales as a model leaves them (every place of every page holds something)."""
    c, kv = _table(case, gen, total), case["kv"]
    for name, (shape, scale_shape) in zip("kv", _pool_shapes(case, c["pages"])):
        if kv == "fp16":
            pool, scales = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float16), None
        elif kv == "int4":
            pool = torch.randint(-(1 << 31), 1 << 31, shape, generator=gen, device="cuda", dtype=torch.int32)
            plain = scale_shape[:4] + scale_shape[5:]                  # (scale, offset) is dimension 4
            s = (torch.rand(plain, generator=gen, device="cuda") * 0.2 + 0.1).half()
            mid = torch.randn(plain, generator=gen, device="cuda") * 0.3   # of the run's values
            scales = torch.stack([s, (mid - 23.5 * s.float()).half()], dim=4).contiguous()
        else:
            if kv == "int8":
                pool = torch.randint(-127, 128, shape, generator=gen, device="cuda", dtype=torch.int8)
            else:
                pool = torch.randint(0, 127, shape, generator=gen, device="cuda", dtype=torch.uint8)        # e4m3, no NaN
                pool += torch.randint(0, 2, shape, generator=gen, device="cuda", dtype=torch.uint8) * 128
            scales = (torch.rand(scale_shape, generator=gen, device="cuda") + 0.5) * (2.0 / QMAX[kv])
        c[name], c[name + "_scales"] = pool, scales
    return c


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    D, Hk = case["head_dim"], case["kv_heads"]
    new, total = _lengths(case)
    half = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").half()  # noqa: E731
    empty = lambda *shape: torch.empty(*shape, dtype=torch.float16, device="cuda")  # noqa: E731
    cache = _cache(case, gen, total)
    tokens = sum(new)
    state = {"case": case, "tokens": tokens, "cu": _ints(_starts(new)), "cache": cache}
    if case["op"] == "append":
        Hq = case["q_heads"]
        state |= {"qkv": half(tokens, (Hq + 2 * Hk) * D), "rope": _rope_table(max(total), case["rotary"]) if case["rotary"] else None,
                  "q_norm": (half(D) * 0.2 + 1) if case["norm"] else None, "k_norm": (half(D) * 0.2 + 1) if case["norm"] else None,
                  "first": _ints([t - n for n, t in zip(new, total)]), "q_out": empty(tokens, Hq, D), "keys": empty(tokens, Hk, D), "values": empty(tokens, Hk, D),
                  "k_out": empty(tokens, Hk, D) if case["new"] > 1 else None}
        return state
    if case["op"] == "evict":
        kept = _kept(case)
        # sums of weights: a few tokens have most, many have little, some exactly the same
        state["scores"] = (torch.rand(cache["pages"], Hk, case["page"], generator=gen, device="cuda") ** 8).half().float()
        to = _table(case, gen, kept)
        for name, (shape, scale_shape) in zip("kv", _pool_shapes(case, to["pages"])):
            to[name] = torch.zeros(shape, dtype=cache[name].dtype, device="cuda")
            to[name + "_scales"] = None if cache[name + "_scales"] is None else torch.zeros(scale_shape, dtype=cache[name + "_scales"].dtype, device="cuda")
        to["lens"] = torch.zeros_like(cache["lens"])
        state |= {"to": to, "to_scores": torch.zeros(to["pages"], Hk, case["page"], device="cuda"), "kept": sum(kept), "cu_kept": _ints(_starts(kept))}
        if case["kv"] != "fp16":
            state |= {"keys": empty(sum(kept), Hk, D), "values": empty(sum(kept), Hk, D)}
    else:
        state["q"] = half(tokens, case["q_heads"], D) * 1.5
        if tokens == case["seqs"] and max(new) == 1:
            state["out"] = torch.empty_like(state["q"])
        if case["op"] == "scores":
            # what the tokens got so far, but for those that are new
            state["earlier"] = torch.rand(cache["pages"], Hk, case["page"], generator=gen, device="cuda") * 4
            state["sums"] = torch.zeros_like(state["earlier"])
    state["workspace"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device="cuda")
    return state


# ---- the plain forms ------------------------------------------------------------------------------------------------------------

def _value(codes, kv):
    return codes.view(torch.float8_e4m3fn).float() if kv == "fp8" else codes.float()


def _code(x, kv):
    """x / scale as the cache holds it."""
    x = x.clamp(-QMAX[kv], QMAX[kv])
    return x.to(torch.float8_e4m3fn).view(torch.uint8) if kv == "fp8" else x.round().to(torch.int8)


def _shifts():
    return torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device="cuda", dtype=torch.int32)


def _pages_plain(cache, table, case, values):
    """Keys or values of whole pages [...][heads][page][dim] in 32 bits, as the cache in 4, 8 or 16 bits holds them."""
    name = "v" if values else "k"
    x, s, kv, D = cache[name][table], cache[name + "_scales"], case["kv"], case["head_dim"]
    if kv == "int4":
        x = ((x[..., None] >> _shifts()) & 15).flatten(-2).float() + 16.0     # keys [..][page][D], values [..][page / 16][D][16]
        s, o = s[table].float().unbind(-2 if values else -1)                  # keys [..][page][G], values [..][page / 16][G][16]
        at = -2 if values else -1
        s, o = (t.repeat_interleave(case["block"], dim=at).narrow(at, 0, D) for t in (s, o))
        x = (x * s + o).half().float()
    else:
        x = _value(x, kv)
    if values:
        x = x.transpose(-1, -2).flatten(-3, -2)
    if kv in QMAX:
        x = x * s[table].repeat_interleave(case["block"], dim=-1)[..., None]
    return x


def _sequences_plain(cache, case):
    """[seqs][heads][places][dim] of keys, and of values"""
    out = []
    for values in (False, True):
        x = _pages_plain(cache, cache["table"].long(), case, values)           # [seqs][pages][heads][page][dim]
        out.append(x.transpose(1, 2).flatten(2, 3))
    return out


def _sequence_of(cu, tokens):
    return torch.searchsorted(cu[1:].contiguous(), torch.arange(tokens, device="cuda", dtype=torch.int32), right=True)


def _plain_norm_rope(x, weight, rope, position, case):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5) * weight.float()
    R = case["rotary"]
    if R == 0:
        return x
    c, s = rope[position, None].unbind(-1)
    if case["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([turned, x[..., R:]], dim=-1)


def _plain_codes(x, case):
    """x [tokens][heads][D] -> codes, and scale and offset [tokens][heads][G]"""
    D, block = case["head_dim"], case["block"]
    pad = -D % block
    runs = lambda fill: torch.nn.functional.pad(x, (0, pad), value=fill).unflatten(-1, (-1, block))  # noqa: E731
    lo, hi = runs(math.inf).amin(-1), runs(-math.inf).amax(-1)
    s = ((hi - lo) * ((1 - 2.0 ** -11) / 15)).half()
    o = (lo - 16 * s.float()).half()
    wide = lambda t: t.float().repeat_interleave(block, dim=-1)[..., :D]  # noqa: E731
    by = torch.where(s > 0, 1 / s.float(), 0.0)
    return ((x - wide(o)) * wide(by) - 16).round().clamp(0, 15).int(), s, o


def _plain_write(state, x, seq, position, values):
    """x [tokens][heads][dim] in 32 bits into the pool of 4 bits."""
    case, cache = state["case"], state["cache"]
    codes, s, o = _plain_codes(x, case)
    page, slot = cache["table"].long()[seq, position // case["page"]], position % case["page"]
    if not values:
        words = (codes.unflatten(-1, (-1, 8)) << _shifts()).sum(-1).to(torch.int32)
        cache["k"][page, :, slot] = words
        cache["k_scales"][page, :, slot] = torch.stack([s, o], dim=-1)
        return
    # a token's four bits within its word: what they change by is added to it, as tokens may share a word
    word, at = slot % 16 // 8, _shifts()[slot % 8][:, None, None]
    old = (cache["v"][page, :, slot // 16, :, word] >> at) & 15
    col = lambda t: t[:, None, None]  # noqa: E731
    heads, dims = torch.arange(case["kv_heads"], device="cuda")[:, None], torch.arange(case["head_dim"], device="cuda")
    cache["v"].index_put_((col(page), heads, col(slot // 16), dims, col(word)), (codes - old) << at, accumulate=True)
    cache["v_scales"][page, :, slot // 16, :, 0, slot % 16] = s
    cache["v_scales"][page, :, slot // 16, :, 1, slot % 16] = o


def _plain_gather(cache, case, cu, first, tokens):
    """[tokens][heads][dim] of keys, and of values"""
    seq = _sequence_of(cu, tokens)
    position = torch.arange(tokens, device="cuda") - cu[seq] + (first[seq] if first is not None else 0)
    keys, values = _sequences_plain(cache, case)
    return [x[seq, :, position].half() for x in (keys, values)]


def _plain_append(state):
    case, cache = state["case"], state["cache"]
    Hq, Hk, D, T = case["q_heads"], case["kv_heads"], case["head_dim"], state["tokens"]
    seq = _sequence_of(state["cu"], T)
    position = cache["lens"].long()[seq] - state["cu"][1:][seq] + torch.arange(T, device="cuda")
    q, k, v = state["qkv"].view(T, Hq + 2 * Hk, D).split([Hq, Hk, Hk], dim=1)
    q = _plain_norm_rope(q, state["q_norm"], state["rope"], position, case)
    k = _plain_norm_rope(k, state["k_norm"], state["rope"], position, case)
    _plain_write(state, k, seq, position, False)
    _plain_write(state, v.float(), seq, position, True)
    out = {"q": q.half(), "k": k.half() if state["k_out"] is not None else []}
    # read back: the token's own place of its page
    page, slot = cache["table"].long()[seq, position // case["page"]], position % case["page"]
    for name, values in (("keys", False), ("values", True)):
        D_run = lambda t: t.float().repeat_interleave(case["block"], dim=-1)[..., :D]  # noqa: E731
        if values:
            word = cache["v"][page, :, slot // 16, :, slot % 16 // 8]
            code = (word >> _shifts()[slot % 8][:, None, None]) & 15
            s, o = (cache["v_scales"][page, :, slot // 16, :, i, slot % 16] for i in (0, 1))
        else:
            code = ((cache["k"][page, :, slot][..., None] >> _shifts()) & 15).flatten(-2)
            s, o = cache["k_scales"][page, :, slot].unbind(-1)
        out[name] = ((code.float() + 16) * D_run(s) + D_run(o)).half()
    return out


def _plain_softmax(scores, seen):
    scores = torch.where(seen, scores, -torch.inf)
    most = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(most == -torch.inf, 0.0, most))
    return p / p.sum(-1, keepdim=True).clamp(min=1e-37)


def _plain_weights(state, keys):
    """Softmax weights [seqs][heads][queries * group][places] of the last queries of every sequence."""
    case, cache = state["case"], state["cache"]
    B, Hk, D = case["seqs"], case["kv_heads"], case["head_dim"]
    cu, lens, n = state["cu"].long(), cache["lens"].long(), 1 if case["op"] == "decode" else case["queries"]
    row = torch.arange(n, device="cuda")
    mine = cu[1:] - cu[:-1]
    q = state["q"].float()[(cu[:-1, None] + row).clamp(max=max(0, state["tokens"] - 1))]              # [seqs][queries][heads][D]
    q = q.view(B, n, Hk, -1, D).permute(0, 2, 1, 3, 4)                                                # [seqs][heads][queries][group][D]
    position = torch.arange(keys.shape[2], device="cuda")
    at = ((lens - mine)[:, None] + row)[..., None]                                                    # of a query
    seen = (position <= at) & (row < mine[:, None])[..., None]
    if case["window"]:
        seen = seen & (position > at - case["window"])
    s = q.reshape(B, Hk, -1, D) @ keys.transpose(-1, -2) * D ** -0.5
    return _plain_softmax(s.unflatten(2, (n, -1)), seen[:, None, :, None]).flatten(2, 3)


def _plain_attention(state, p, values):
    case, cache = state["case"], state["cache"]
    held = torch.arange(values.shape[2], device="cuda") < cache["lens"][:, None]
    return (p @ torch.where(held[:, None, :, None], values, 0.0)).half().view(case["seqs"], -1, case["head_dim"])


def _plain_sums(state, p):
    """What every cached token has got, after what it had before this call's tokens; zeros where no token is."""
    case, cache = state["case"], state["cache"]
    page, L = case["page"], p.shape[-1]
    position, table = torch.arange(L, device="cuda"), cache["table"].long()
    at = table[:, position // page][:, None] * (case["kv_heads"] * page) + torch.arange(case["kv_heads"], device="cuda")[:, None] * page + position % page
    had = position < (cache["lens"].long() - (state["cu"][1:] - state["cu"][:-1]))[:, None]
    sums = p.sum(2)
    if case["queries"] == 1:
        sums = sums + torch.where(had[:, None], state["earlier"].flatten()[at], 0.0)
    held = (position < cache["lens"][:, None])[:, None].expand(at.shape)
    out = torch.zeros(state["earlier"].numel() + 1, device="cuda")
    out[torch.where(held, at, state["earlier"].numel())] = torch.where(held, sums, 0.0)
    return out[:-1].view_as(state["earlier"])


def _plain_scores(state):
    keys, values = _sequences_plain(state["cache"], state["case"])
    p = _plain_weights(state, keys)
    out = {"sums": _plain_sums(state, p)}
    if state["case"]["queries"] == 1:
        out["out"] = _plain_attention(state, p, values)
    return out


def _plain_evict(state):
    case, cache, to = state["case"], state["cache"], state["to"]
    B, H, D, page, kv, block, budget = case["seqs"], case["kv_heads"], case["head_dim"], case["page"], case["kv"], case["block"], case["budget"]
    L, M = cache["most"] * page, to["most"] * page
    position, lens = torch.arange(L, device="cuda"), cache["lens"].long()
    scores = state["scores"][cache["table"].long()].transpose(1, 2).flatten(2, 3)                     # [seqs][heads][places]
    held = (position < lens[:, None])[:, None]
    always = (position < case["first"]) | (position >= lens[:, None] - case["last"])
    rank = torch.where(held, torch.where(always[:, None], torch.inf, scores), -torch.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :budget]
    kept = lens.clamp(max=budget)
    place = torch.arange(order.shape[-1], device="cuda")
    taken = (place < kept[:, None])[:, None]
    source = torch.where(taken, order, L).sort(dim=-1).values                                         # in order; L: none
    source = torch.nn.functional.pad(source, (0, M - source.shape[-1]), value=L) if M > source.shape[-1] else source[..., :M]
    taken, source, place = source < L, source.clamp(max=L - 1), torch.arange(M, device="cuda")
    head = torch.arange(H, device="cuda")[:, None]
    from_page = torch.gather(cache["table"].long()[:, None].expand(B, H, -1), 2, source // page)
    to_page = to["table"].long()[:, None, place // page].expand(B, H, M)
    to_page = torch.where(taken, to_page, to["pages"])                                                # past the pool: nowhere
    a, b = source % page, place % page
    grown = lambda t: torch.cat([t, torch.zeros_like(t[:1])])  # noqa: E731  with a page that takes what goes nowhere
    out = {"lens": kept.int()}
    sums = grown(torch.zeros_like(state["to_scores"]))
    sums[to_page, head, b] = state["scores"][from_page, head, a]
    out["scores"] = sums[:-1]
    made = {}
    for name in "kv":
        old, new = cache[name], grown(torch.zeros_like(to[name]))
        old_s, new_s = cache[name + "_scales"], None if cache[name + "_scales"] is None else grown(torch.zeros_like(to[name + "_scales"]))
        values = name == "v"
        if kv == "int4":
            if values:
                code = (old[from_page, head, a // 16, :, a % 16 // 8] >> _shifts()[a % 8][..., None]) & 15
                whole = torch.zeros(new.shape[:-1] + (16,), dtype=torch.int32, device="cuda")
                whole[to_page, head, b // 16, :, b % 16] = code
                new = (whole.unflatten(-1, (2, 8)) << _shifts()).sum(-1).to(torch.int32)
                for i in (0, 1):
                    new_s[to_page, head, b // 16, :, i, b % 16] = old_s[from_page, head, a // 16, :, i, a % 16]
            else:
                new[to_page, head, b] = old[from_page, head, a]
                new_s[to_page, head, b] = old_s[from_page, head, a]
        else:
            x = old[from_page, head, a // 16, :, a % 16] if values else old[from_page, head, a]
            if kv != "fp16":
                # a block has the largest scale of what comes into it
                mine = torch.where(taken, old_s[from_page, head, a // block], 0.0)
                most = mine.unflatten(-1, (-1, block)).amax(-1).repeat_interleave(block, dim=-1)
                again = _code(_value(x, kv) * torch.where(most > 0, mine / most, 0.0)[..., None], kv)
                x = torch.where((mine == most)[..., None], x, again)
                new_s[to_page, head, b // block] = most
            if values:
                new[to_page, head, b // 16, :, b % 16] = x
            else:
                new[to_page, head, b] = x
        made[name], made[name + "_scales"] = new[:-1], None if new_s is None else new_s[:-1]
    if kv == "fp16":
        return out | {"keys": made["k"], "values": made["v"]}
    out["keys"], out["values"] = _plain_gather(to | made, case, state["cu_kept"], None, state["kept"])
    return out


# ---- the framework's calls ------------------------------------------------------------------------------------------------------

def _bind(state):
    """The descriptors that a program keeps beside its buffers."""
    import paper_2512_17970_amd as cg
    case, calls = state["case"], {"cg": cg}
    D, Hk = case["head_dim"], case["kv_heads"]

    def cache(c):
        return cg.KvCache.make(c["k"], c["v"], c["k_scales"], c["v_scales"], c["table"], c["lens"], kv_heads=Hk, head_dim=D, num_pages=c["pages"],
                               page_size=case["page"], dtype=KV_TYPES[case["kv"]], scale_block=case["block"], num_seqs=case["seqs"], max_pages=c["most"])
    calls["cache"] = cache(state["cache"])
    if case["op"] == "append":
        Hq, qkv = case["q_heads"], state["qkv"]
        calls["desc"] = cg.AppendDesc.make(state["tokens"], Hq, rotary_dim=case["rotary"], rope_positions=0 if state["rope"] is None else state["rope"].shape[0],
                                           interleaved=case["interleaved"], norm_eps=1e-5, q_stride=qkv.shape[1], k_stride=qkv.shape[1], v_stride=qkv.shape[1])
        calls["qkv"] = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D], qkv[:, (Hq + Hk) * D:]
    elif case["op"] == "evict":
        calls["to"] = cache(state["to"])
        calls["desc"] = cg.EvictDesc.make(case["budget"], keep_first=case["first"], keep_last=case["last"], max_kv=case["longest"])
    else:
        calls["desc"] = cg.AttnDesc.make(case["q_heads"], Hk, D, num_seqs=case["seqs"], total_q=state["tokens"], max_kv=case["longest"], scale=D ** -0.5,
                                         window=case["window"])
    return calls


def _own(state):
    if "calls" not in state:
        state["calls"] = _bind(state)
    calls, case = state["calls"], state["case"]
    cg, stream = calls["cg"], torch.cuda.current_stream().cuda_stream
    cache, desc = calls["cache"], calls["desc"]
    if case["op"] == "append":
        q, k, v = calls["qkv"]
        cg.codegemm_kv_append(cache, desc, state["cu"], q, k, v, state["q_norm"], state["k_norm"], state["rope"], state["q_out"], state["k_out"], stream)
        cg.codegemm_kv_gather(cache, state["tokens"], state["cu"], state["first"], state["keys"], state["values"], stream)
        return {"q": state["q_out"], "k": state["k_out"] if state["k_out"] is not None else [], "keys": state["keys"], "values": state["values"]}
    if case["op"] == "decode":
        cg.codegemm_attn_decode(cache, desc, state["q"], state["out"], state["workspace"], WORKSPACE, stream)
        return state["out"]
    if case["op"] == "scores":
        if case["queries"] == 1:
            cg.codegemm_attn_decode_scores(cache, desc, state["q"], state["out"], None, state["earlier"], state["sums"], state["workspace"], WORKSPACE, stream)
            return {"sums": state["sums"], "out": state["out"]}
        if state["tokens"]:
            cg.codegemm_attn_scores(cache, desc, state["q"], state["cu"], None, None, state["sums"], state["workspace"], WORKSPACE, stream)
        return {"sums": state["sums"]}
    to = state["to"]
    cg.codegemm_kv_evict(cache, calls["to"], desc, state["scores"], None, state["to_scores"], to["lens"], None, state["workspace"], WORKSPACE, stream)
    if case["kv"] == "fp16":
        return {"lens": to["lens"], "scores": state["to_scores"], "keys": to["k"], "values": to["v"]}
    cg.codegemm_kv_gather(calls["to"], state["kept"], state["cu_kept"], None, state["keys"], state["values"], stream)
    return {"lens": to["lens"], "scores": state["to_scores"], "keys": state["keys"], "values": state["values"]}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "append":
        return _plain_append(state)
    if op == "scores":
        return _plain_scores(state)
    if op == "evict":
        return _plain_evict(state)
    keys, values = _sequences_plain(state["cache"], state["case"])
    return _plain_attention(state, _plain_weights(state, keys), values)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------------

def work(case):
    D, Hk, kv = case["head_dim"], case["kv_heads"], case["kv"]
    new, total = _lengths(case)
    T = sum(new)
    # keys (or values) of n tokens with their scales
    held = lambda n: Hk * (2 * n * D if kv == "fp16" else n * D // 2 + 4 * n * _runs(case) if kv == "int4" else n * D + 4 * -(-n // case["block"]))  # noqa: E731
    if case["op"] == "append":
        Hq = case["q_heads"]
        rope = 4 * case["rotary"] * (min(T, max(total)) if case["rotary"] else 0)
        return {"bytes": 2 * T * D * (Hq + 2 * Hk + Hq + (Hk if case["new"] > 1 else 0)) + rope + sum(2 * 2 * held(n) for n in new) + 4 * Hk * D * T,
                "flops": T * D * (Hq + 2 * Hk) * 3}
    if case["op"] == "evict":
        kept = _kept(case)
        read = 0 if kv == "fp16" else sum(2 * held(n) for n in kept) + 4 * Hk * D * sum(kept)
        return {"bytes": 4 * Hk * sum(total) + sum(4 * held(n) for n in kept) + 4 * Hk * sum(kept) + read, "flops": Hk * sum(total)}
    Hq, W = case["q_heads"], case["window"]
    keys = [min(t, W + n - 1) if W else t for n, t in zip(new, total)]
    if case["op"] == "decode":
        return {"bytes": sum(2 * held(n) for n in keys) + 4 * case["seqs"] * Hq * D, "flops": 4 * Hq * D * sum(keys)}
    single = case["queries"] == 1
    pairs = sum(n * min(t, W) if W else n * t - n * (n - 1) // 2 for n, t in zip(new, total))
    return {"bytes": sum((2 if single else 1) * held(n) for n in keys) + (8 if single else 4) * Hk * sum(total) + 2 * (2 if single else 1) * T * Hq * D,
            "flops": (4 if single else 2) * Hq * D * pairs}


# ---- the definitions in 64 bits, sequence by sequence ------------------------------------------------------------------------------

def _exact_nibbles(words):
    """The eight codes of a word, in order: low and high half in turn."""
    w = words.long() & 0xFFFFFFFF
    return torch.stack([torch.div(w, 1 << (4 * (j // 2) + 16 * (j % 2)), rounding_mode="floor") % 16 for j in range(8)], dim=-1)


def _exact_tokens(case, c, i, n, values):
    """Keys or values [n][heads][dim] of sequence i as its cache holds them, in 64 bits."""
    pool, scales = (c["v"], c["v_scales"]) if values else (c["k"], c["k_scales"])
    p = torch.arange(n, device="cuda")
    page, slot = c["table"][i].long()[p // case["page"]], p % case["page"]
    if case["kv"] != "int4":
        x = _value(pool[page, :, slot // 16, :, slot % 16] if values else pool[page, :, slot], case["kv"]).double()
        return x if scales is None else x * scales[page, :, slot // case["block"]].double()[..., None]
    run = torch.arange(case["head_dim"], device="cuda") // case["block"]
    if values:
        eight = _exact_nibbles(pool[page, :, slot // 16, :, slot % 16 // 8])
        code = torch.gather(eight, -1, (slot % 8)[:, None, None, None].expand(*eight.shape[:-1], 1))[..., 0]
        s, o = (scales[page, :, slot // 16, :, k, slot % 16].double()[..., run] for k in (0, 1))
    else:
        code = _exact_nibbles(pool[page, :, slot]).flatten(-2)
        s, o = (scales[page, :, slot, :, k].double()[..., run] for k in (0, 1))
    return ((code.double() + 16) * s + o).half().double()               # a cached value is a number in fp16


def _exact_rope(x, weight, positions, case):
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + 1e-5) * weight.double()
    R = case["rotary"]
    if R:
        # the table's own values: they are an input
        t = _rope_table(int(positions.max()) + 1, R)[positions].double()
        z = torch.complex(t[..., 0], t[..., 1])[:, None]
        pair = x[..., :R].unflatten(-1, (-1, 2)) if case["interleaved"] else x[..., :R].unflatten(-1, (2, -1)).transpose(-1, -2)
        turned = torch.view_as_real(torch.complex(pair[..., 0].contiguous(), pair[..., 1].contiguous()) * z)
        x = torch.cat([turned.flatten(-2) if case["interleaved"] else turned.transpose(-1, -2).flatten(-2), x[..., R:]], dim=-1)
    return x


def _exact_four_bits(x, case):
    """What a cache in 4 bits holds for x, run by run of its dimensions."""
    out = []
    for run in x.split(case["block"], dim=-1):
        lo, hi = run.min(-1, keepdim=True).values, run.max(-1, keepdim=True).values
        s = ((hi - lo) * (1 - 2.0 ** -11) / 15).half().double()
        o = (lo - 16 * s).half().double()
        code = torch.where(s > 0, torch.round((run - o) / torch.where(s > 0, s, 1.0) - 16).clamp(0, 15), 0.0)
        out.append(((code + 16) * s + o).half().double())
    return torch.cat(out, dim=-1)


def _exact_append(state):
    case = state["case"]
    Hq, Hk, D = case["q_heads"], case["kv_heads"], case["head_dim"]
    new, total = _lengths(case)
    out, at = {"q": [], "k": [], "keys": [], "values": []}, 0
    for n, t in zip(new, total):
        rows = state["qkv"][at:at + n].double()
        at += n
        q, k, v = rows[:, :Hq * D].view(n, Hq, D), rows[:, Hq * D:(Hq + Hk) * D].view(n, Hk, D), rows[:, (Hq + Hk) * D:].view(n, Hk, D)
        positions = torch.arange(t - n, t, device="cuda")
        q, k = _exact_rope(q, state["q_norm"], positions, case), _exact_rope(k, state["k_norm"], positions, case)
        for name, x in (("q", q), ("k", k), ("keys", _exact_four_bits(k, case)), ("values", _exact_four_bits(v, case))):
            out[name].append(x)
    out = {name: torch.cat(x) for name, x in out.items()}
    return out if state["k_out"] is not None else out | {"k": []}


def _exact_sequence(case, state, i, n, at, rows):
    """Softmax weights' sums [heads][n], and the attention of the queries [rows][q heads][D], of one sequence of n tokens."""
    k, v = (_exact_tokens(case, state["cache"], i, n, values) for values in (False, True))
    q, D, Hk = state["q"][at:at + rows].double(), case["head_dim"], case["kv_heads"]
    group = case["q_heads"] // Hk
    key, query = torch.arange(n, device="cuda"), torch.arange(n - rows, n, device="cuda")[:, None]
    hidden = key > query
    if case["window"]:
        hidden = hidden | (key <= query - case["window"])
    sums, out = torch.zeros(Hk, n, dtype=torch.float64, device="cuda"), torch.zeros_like(q)
    for h in range(case["q_heads"]):
        s = (q[:, h] @ k[:, h // group].t() / math.sqrt(D)).masked_fill(hidden, -math.inf)
        p = torch.softmax(s, dim=-1)
        sums[h // group] += p.sum(0)
        out[:, h] = p @ v[:, h // group]
    return sums, out


def _exact_evicted(state, i, n, h):
    """Positions that sequence i keeps of key head h."""
    case, c = state["case"], state["cache"]
    p = torch.arange(n, device="cuda")
    if n <= case["budget"]:
        return p
    score = state["scores"][c["table"][i].long()[p // case["page"]], h, p % case["page"]].double()
    lo, hi = case["first"], n - case["last"]
    room, keep = case["budget"] - lo - case["last"], torch.ones(n, dtype=torch.bool, device="cuda")
    between = score[lo:hi]
    if room == 0:
        keep[lo:hi] = False
    else:
        least = between.kthvalue(hi - lo - room + 1).values
        above, same = between > least, between == least
        keep[lo:hi] = above | (same & (same.cumsum(0) <= room - above.sum()))
    return p[keep]


def _exact_evict(state):
    case, to, H = state["case"], state["to"], state["case"]["kv_heads"]
    kv, block, page = case["kv"], case["block"], case["page"]
    total, kept = _lengths(case)[1], _kept(case)
    scores = torch.zeros(to["pages"], H, page, dtype=torch.float64, device="cuda")
    rows = {"k": [], "v": []}
    for i, (n, m) in enumerate(zip(total, kept)):
        if n == 0:
            continue
        table, t = state["cache"]["table"][i].long(), torch.arange(m, device="cuda")
        source = [_exact_evicted(state, i, n, h) for h in range(H)]
        for h in range(H):
            scores[to["table"][i].long()[t // page], h, t % page] = state["scores"][table[source[h] // page], h, source[h] % page].double()
        for name in "kv":
            x = _exact_tokens(case, state["cache"], i, n, name == "v")
            mine = torch.stack([x[source[h], h] for h in range(H)], dim=1)
            if kv in QMAX:                                             # blocks of the largest scale
                s = state["cache"][name + "_scales"]
                old = torch.stack([s[table[source[h] // page], h, source[h] % page // block].double() for h in range(H)], dim=1)
                pad = -m % block
                most = torch.nn.functional.pad(old, (0, 0, 0, pad)).unflatten(0, (-1, block)).amax(1).repeat_interleave(block, dim=0)[:m]
                codes = mine / most[..., None]
                mine = torch.where((old == most)[..., None], mine, _value(_code(codes.float() if kv == "fp8" else codes, kv), kv).double() * most[..., None])
            rows[name].append(mine)
    out = {"lens": None, "scores": scores}
    for name, key in (("k", "keys"), ("v", "values")):
        if kv != "fp16":
            out[key] = torch.cat(rows[name])
            continue
        pool, at = torch.zeros_like(to[name]).double(), 0
        for i, m in enumerate(x for x in kept):
            if m == 0:
                continue
            t = torch.arange(m, device="cuda")
            where = to["table"][i].long()[t // page]
            if name == "v":
                pool[where, :, t % page // 16, :, t % 16] = rows[name][at]
            else:
                pool[where, :, t % page] = rows[name][at]
            at += 1
        out[key] = pool
    return out


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(state)
    if case["op"] == "evict":
        return _exact_evict(state)
    new, total = _lengths(case)
    if case["q_heads"] * sum(n * t for n, t in zip(new, total)) * case["head_dim"] > 1 << 40:
        return None
    outs, c = [], state["cache"]
    sums = torch.zeros(c["pages"], case["kv_heads"], case["page"], dtype=torch.float64, device="cuda")
    at = 0
    for i, (rows, n) in enumerate(zip(new, total)):
        if n == 0:
            outs.append(torch.zeros(rows, case["q_heads"], case["head_dim"], dtype=torch.float64, device="cuda"))
            at += rows
            continue
        got, out = _exact_sequence(case, state, i, n, at, rows)
        at += rows
        outs.append(out)
        t = torch.arange(n, device="cuda")
        page, slot = c["table"][i].long()[t // case["page"]], t % case["page"]
        if case["op"] == "scores":
            had = state["earlier"][page, :, slot].double().t() * (t < n - rows) if case["queries"] == 1 else 0.0
            sums[page, :, slot] = (got + had).t()
    if case["op"] == "decode":
        return torch.cat(outs)
    return {"sums": sums, "out": torch.cat(outs)} if case["queries"] == 1 else {"sums": sums}

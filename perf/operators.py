"""Cases of the operators on device tensors: a key/value cache and the attentions beside it.

  store    ss_cache_write, ss_cache_read: keys and values of listed tokens are written to their slots of a cache (held in 8
           bits with one scale per vector, or in 16), and read back as the values that the cache stands for.
  tree     ss_attention_tree: nodes of a drafted tree (or single tokens, the decode step) attend to their sequence's cache and,
           as far as their mask says, to each other.  The nodes' keys and values are in the cache already, behind the context.
  packed   ss_attention_packed: causal attention of whole prompts that lie behind each other without padding.

Widths are those of this repository's models (4 heads of 64; 32 and 40 heads of 128), and 32 or 64 heads that share 4 or 8
key/value heads.  Lengths go from one token to tens of thousands; sequences of a case differ in length, by a law that the
case's own numbers fix (so that `work` can count), whereas the seed makes the values, the trees and the places in the cache.

A cache holds for each sequence a slab of slots: element e of the vector of head h in slot s of sequence i lies at
(start[i] * heads + h * slots[i] + s) * dim + e.  In 8 bits a vector is round(x / scale), scale = max|x| / 127.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}
SIZE = {"f16": 2, "bf16": 2, "i8": 1}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token of one row of the small test model enters its cache
        dict(name="store_one_token", op="store", seqs=1, tokens=1, context=40, kv_heads=4, dim=64, type="f16", cache="i8"),
        # a decode step of 64 rows with shared heads: one token each, at places all over the cache
        dict(name="store_step_64", op="store", seqs=64, tokens=1, context=4000, kv_heads=8, dim=128, type="bf16", cache="i8"),
        # the keys and values of a prompt forward, a group of prompts at the 7B widths
        dict(name="store_prompts_7b", op="store", seqs=128, tokens=180, context=0, kv_heads=32, dim=128, type="f16", cache="i8"),
        # decode step of 16 rows at short contexts, 7B widths, cache in 16 bits
        dict(name="step_16_short_7b", op="tree", seqs=16, nodes=1, context=250, heads=32, kv_heads=32, dim=128, type="f16", cache="f16"),
        # one row late in a long answer at the 7B widths, cache in 8 bits: the smallest call, all latency
        dict(name="step_1_long_7b", op="tree", seqs=1, nodes=1, context=3900, heads=32, kv_heads=32, dim=128, type="f16", cache="i8"),
        # decode step of 64 rows with shared heads at contexts up to 8000, cache in 8 bits: bound by the cache's bytes
        dict(name="step_64_shared", op="tree", seqs=64, nodes=1, context=8000, heads=32, kv_heads=8, dim=128, type="bf16", cache="i8"),
        # sixteen drafted nodes for one answer at the 13B widths
        dict(name="draft_16_of_1_13b", op="tree", seqs=1, nodes=16, context=701, heads=40, kv_heads=40, dim=128, type="f16", cache="f16"),
        # trees of up to 61 nodes for eight rows with shared heads, long contexts
        dict(name="draft_61_of_8_shared", op="tree", seqs=8, nodes=61, context=6000, heads=32, kv_heads=8, dim=128, type="bf16", cache="i8"),
        # prompts of the small test model
        dict(name="packed_tiny", op="packed", seqs=16, tokens=32, heads=4, kv_heads=4, dim=64, type="f16"),
        # a group of short prompts at the 7B widths
        dict(name="packed_group_7b", op="packed", seqs=256, tokens=256, heads=32, kv_heads=32, dim=128, type="f16"),
        # a few long prompts, shared heads
        dict(name="packed_long_shared", op="packed", seqs=6, tokens=4001, heads=32, kv_heads=8, dim=128, type="bf16"),
        # one prompt of 12288 tokens, shared heads
        dict(name="packed_one_shared", op="packed", seqs=1, tokens=12288, heads=32, kv_heads=8, dim=128, type="bf16"),
    ]


def draw(rng):
    def upto(lo, hi):   # spread over the logarithm
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(("store", "tree", "tree", "packed"))
        kv, group = rng.choice(((4, 1), (32, 1), (40, 1), (1, 8), (2, 4), (8, 4), (8, 8), (4, 7)))
        c = dict(op=op, kv_heads=kv, dim=rng.choice((64, 128, 128)), type=rng.choice(("f16", "bf16")))
        if op == "store":
            c.update(seqs=upto(1, 256), tokens=rng.choice((1, upto(1, 2000))), context=rng.choice((0, upto(1, 4000))), cache=rng.choice(("i8", "i8", c["type"])))
        elif op == "tree":
            c.update(heads=kv * group, seqs=upto(1, 100), nodes=rng.choice((1, upto(2, 64))), context=upto(1, 30000), cache=rng.choice(("i8", "i8", c["type"])))
        else:
            c.update(heads=kv * group, seqs=upto(1, 300), tokens=upto(1, 12000))
        w = work(c)
        if w["bytes"] <= 1e9 and w["flops"] <= 1.2e12 and _padded(c) <= (4.8e9 if op == "packed" else 2.5e9):
            return c


def _padded(c):
    """Values that the plain form's largest tables hold."""
    if c["op"] == "store":
        return c["seqs"] * (c["context"] + c["tokens"]) * c["kv_heads"] * c["dim"]
    if c["op"] == "tree":
        n = c["seqs"] * (c["context"] + c["nodes"])
        return n * max(c["kv_heads"] * c["dim"], c["heads"] * c["nodes"])
    return c["seqs"] * c["tokens"] * max(c["tokens"], c["dim"]) * c["heads"]


def _lengths(n, top, least, law):
    """n lengths from `least` to `top`, of which one is `top`: from short to long without an order, most of them short."""
    r = random.Random(1000 * n + top + law)
    got = [least + int((top - least) * r.random() ** 1.5) for _ in range(n)]
    got[r.randrange(n)] = top
    return got


def _shape(c):
    """Contexts and counts of tokens (or nodes) of a case's sequences."""
    n = c["seqs"]
    if c["op"] == "packed":
        return [0] * n, _lengths(n, c["tokens"], 1, 1)
    new = _lengths(n, c["tokens" if c["op"] == "store" else "nodes"], 1, 1)
    return _lengths(n, c["context"], min(c["context"], 1), 2), new


def work(case):
    ctx, new = _shape(case)
    c, tokens = case, sum(new)
    if c["op"] == "store":   # keys and values come in, lie in the cache, and go out
        n = 2 * tokens * c["kv_heads"]
        return {"bytes": n * (c["dim"] * (4 + SIZE[c["cache"]]) + (4 if c["cache"] == "i8" else 0)) + 8 * tokens, "flops": 4 * n * c["dim"]}
    rows = 2 * tokens * c["heads"] * c["dim"] * SIZE[c["type"]]   # queries and results
    if c["op"] == "packed":
        pairs = sum(n * (n + 1) // 2 for n in new)
        return {"bytes": rows + 2 * tokens * c["kv_heads"] * c["dim"] * SIZE[c["type"]], "flops": 4 * pairs * c["heads"] * c["dim"]}
    slots = sum(ctx) + tokens
    pairs = sum(a * b + b for a, b in zip(ctx, new))   # of a node's visible nodes only itself is sure
    return {"bytes": rows + 2 * slots * c["kv_heads"] * (c["dim"] * SIZE[c["cache"]] + (4 if c["cache"] == "i8" else 0)), "flops": 4 * pairs * c["heads"] * c["dim"]}


# ------------------------------------------------------------------------------------------------ inputs
def _vectors(g, n, heads, dim, dtype):
    """Keys, values or queries: normal, with channels of different size, as projections have them."""
    gain = torch.exp(0.4 * torch.randn(heads, dim, device="cuda", generator=g))
    return (torch.randn(n, heads, dim, device="cuda", generator=g) * gain).to(dtype)


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _tree(rng, n, words):
    """Visible nodes of each node of a random tree, as bits: itself, its parent and what the parent sees."""
    bits = []
    for t in range(n):
        up = rng.randrange(-1, t) if t else -1
        bits.append((bits[up] if up >= 0 else 0) | 1 << t)
    return [[(b >> 64 * w & 2**64 - 1) - (1 << 64) * (b >> 64 * w + 63 & 1) for w in range(words)] for b in bits]


def prepare(case, seed):
    c, dtype = case, TYPES[case["type"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    ctx, new = _shape(c)
    n, tokens = c["seqs"], sum(new)
    s = {"case": c}
    if c["op"] == "packed":
        s["q"] = _vectors(g, tokens, c["heads"], c["dim"], dtype)
        s["k"], s["v"] = (_vectors(g, tokens, c["kv_heads"], c["dim"], dtype) for _ in range(2))
        s["offsets"] = _ints(np.concatenate([[0], np.cumsum(new)]).tolist())
        s["max_len"] = max(new)
        return s
    slots = [a + b + rng.randrange(40) for a, b in zip(ctx, new)]   # some room behind each sequence
    order = list(range(n))
    rng.shuffle(order)                                              # and no order among the slabs
    start, at = [0] * n, 0
    for i in order:
        start[i], at = at, at + slots[i]
    s.update(start=_ints(start, torch.int64), slots=_ints(slots), total=at)
    width = c["kv_heads"] * c["dim"]
    if c["op"] == "store":
        s["k_cache"], s["v_cache"] = (torch.zeros(at * width, dtype=TYPES[c["cache"]], device="cuda") for _ in range(2))
        s["k_scale"], s["v_scale"] = (torch.zeros(at * c["kv_heads"], device="cuda") if c["cache"] == "i8" else None for _ in range(2))
        s["k"], s["v"] = (_vectors(g, tokens, c["kv_heads"], c["dim"], dtype) for _ in range(2))
        s["seq"] = _ints(np.repeat(np.arange(n), new).tolist())
        s["slot"] = _ints(np.concatenate([a + np.arange(b) for a, b in zip(ctx, new)]).tolist())
        return s
    if c["cache"] == "i8":   # a whole cache of stored vectors: their codes reach 127, their scales are those of the channels above
        for name in ("k", "v"):
            x = _vectors(g, at, c["kv_heads"], c["dim"], torch.float32)
            scale = x.abs().amax(-1, keepdim=True) / 127
            s[name + "_cache"], s[name + "_scale"] = torch.round(x / scale).to(torch.int8).reshape(-1), scale.reshape(-1)
            del x
    else:
        s["k_cache"], s["v_cache"] = (_vectors(g, at, c["kv_heads"], c["dim"], dtype).reshape(-1) for _ in range(2))
        s["k_scale"] = s["v_scale"] = None
    s["q"] = _vectors(g, tokens, c["heads"], c["dim"], dtype)
    s["context"] = _ints(ctx)
    s["nodes"] = _ints(np.concatenate([[0], np.cumsum(new)]).tolist())
    s["max_context"], s["max_nodes"] = c["context"], c["nodes"]
    s["mask"] = None
    if c["nodes"] > 1:
        words = (c["nodes"] + 63) // 64
        s["mask"] = _ints([row for b in new for row in _tree(rng, b, words)], torch.int64)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c)
    return {"store": _plain_store, "tree": _plain_tree, "packed": _plain_packed}[c["op"]](s, c)


def _own(s, c):
    from paper_2305_13144_amd import binding as ss

    if c["op"] == "packed":
        return ss.ss_attention_packed(s["q"], s["k"], s["v"], s["offsets"], s["max_len"])
    if "handle" not in s:   # what a program keeps with its cache: a view of the tensors, nothing computed
        s["handle"] = ss.Cache(s["k_cache"], s["v_cache"], s["start"], s["slots"], c["kv_heads"], c["dim"], s["k_scale"], s["v_scale"])
    if c["op"] == "store":
        ss.ss_cache_write(s["handle"], s["k"], s["v"], s["seq"], s["slot"])
        return ss.ss_cache_read(s["handle"], s["seq"], s["slot"], s["k"].dtype)
    if c["nodes"] == 1:   # the decode step: a token a row
        return ss.ss_attention_tree(s["q"], s["handle"], s["context"], s["max_context"])
    return ss.ss_attention_tree(s["q"], s["handle"], s["context"], s["max_context"], nodes=s["nodes"], max_nodes=s["max_nodes"], mask=s["mask"])


def _vector_of(s, c, seq, slot):
    """Number of the vector of each head in the given slots: [..., heads]."""
    head = torch.arange(c["kv_heads"], device="cuda")
    seq = seq.long()
    return (s["start"][seq] * c["kv_heads"]).unsqueeze(-1) + head * s["slots"][seq].long().unsqueeze(-1) + slot.long().unsqueeze(-1)


def _held(s, c, name, at):
    x = s[name + "_cache"].view(-1, c["dim"])[at].float()
    return x * s[name + "_scale"][at].unsqueeze(-1) if c["cache"] == "i8" else x


def _plain_store(s, c):
    at = _vector_of(s, c, s["seq"], s["slot"])

    def write(name):
        x = s[name].float()
        if c["cache"] == "i8":
            scale = x.abs().amax(-1) / 127
            x = torch.where(scale.unsqueeze(-1) > 0, torch.round(x / scale.unsqueeze(-1)), 0.0)
            s[name + "_scale"][at] = scale
        s[name + "_cache"].view(-1, c["dim"])[at] = x.to(TYPES[c["cache"]])
        return _held(s, c, name, at).to(s[name].dtype)

    return write("k"), write("v")


def _softmax_product(scores, visible, v):
    """Weights of the visible slots, whose sum is one, times their values; zero where nothing is visible."""
    scores = scores.masked_fill(~visible, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(scores - top)
    return torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp_min(1e-38)


def _plain_tree(s, c):
    n, top, nodes, kv, hd = c["seqs"], c["context"] + c["nodes"], c["nodes"], c["kv_heads"], c["dim"]
    group = c["heads"] // kv
    count = (s["nodes"][1:] - s["nodes"][:-1]).long()
    slot = torch.arange(top, device="cuda")
    at = _vector_of(s, c, torch.arange(n, device="cuda").unsqueeze(-1), torch.minimum(slot, s["slots"].long().unsqueeze(-1) - 1))
    at = at.transpose(1, 2)                                                                   # [n, kv, top]
    t = torch.arange(nodes, device="cuda")
    row = torch.minimum(s["nodes"][:-1].long().unsqueeze(-1) + t, s["nodes"][1:].long().unsqueeze(-1) - 1)   # [n, nodes]
    q = s["q"][row].float().view(n, nodes, kv, group, hd).permute(0, 2, 1, 3, 4).reshape(n, kv, nodes * group, hd)
    scores = torch.matmul(q, _held(s, c, "k", at).transpose(2, 3).contiguous()) * hd ** -0.5
    behind = slot - s["context"].long().unsqueeze(-1)                                         # [n, top]: number of the node in a slot
    if s["mask"] is None:
        drafted = behind.unsqueeze(1) <= t.unsqueeze(-1)
    else:
        word = s["mask"][row].gather(2, (behind.clamp(0, nodes - 1) >> 6).unsqueeze(1).expand(n, nodes, top))
        drafted = (word >> (behind.clamp_min(0) & 63).unsqueeze(1)) & 1 == 1
        drafted = drafted & (behind < count.unsqueeze(-1)).unsqueeze(1)
    visible = (behind < 0).unsqueeze(1) | drafted                                             # [n, nodes, top]
    visible = visible.unsqueeze(2).expand(n, nodes, group, top).reshape(n, 1, nodes * group, top)
    out = _softmax_product(scores, visible, _held(s, c, "v", at))
    out = out.view(n, kv, nodes, group, hd).permute(0, 2, 1, 3, 4).reshape(n, nodes, c["heads"], hd)
    return out[t < count.unsqueeze(-1)].to(s["q"].dtype)


def _plain_packed(s, c):
    n, top, kv, hd = c["seqs"], c["tokens"], c["kv_heads"], c["dim"]
    group = c["heads"] // kv
    t = torch.arange(top, device="cuda")
    first, end = s["offsets"][:-1].long().unsqueeze(-1), s["offsets"][1:].long().unsqueeze(-1)
    row = torch.minimum(first + t, end - 1)
    q = s["q"][row].float().view(n, top, kv, group, hd).permute(0, 2, 3, 1, 4).contiguous()
    k = s["k"][row].float().permute(0, 2, 3, 1).unsqueeze(2).contiguous()
    v = s["v"][row].float().permute(0, 2, 1, 3).unsqueeze(2).contiguous()
    out = _softmax_product(torch.matmul(q, k) * hd ** -0.5, t <= t.unsqueeze(-1), v)          # [n, kv, group, top, hd]
    return out.permute(0, 3, 1, 2, 4).reshape(n, top, c["heads"], hd)[first + t < end].to(s["q"].dtype)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s, c = prepare(case, seed), case
    kv, hd = c["kv_heads"], c["dim"]
    if c["op"] == "store":
        def stored(x):
            x = x.double()
            if c["cache"] != "i8":
                return x
            unit = x.abs().max(dim=2, keepdim=True).values / 127
            return torch.where(unit > 0, (x / unit).round() * unit, x)
        return stored(s["k"]), stored(s["v"])
    group = c["heads"] // kv
    ctx, new = _shape(c)
    out = torch.empty(sum(new), c["heads"], hd, dtype=torch.float64, device="cuda")
    first = 0
    for i in range(c["seqs"]):
        n = new[i]
        if c["op"] == "packed":
            k, v = (s[m][first:first + n].transpose(0, 1).double() for m in ("k", "v"))
            hidden = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
        else:
            size, a = int(s["slots"][i]), int(s["start"][i]) * kv

            def part(m):
                x = s[m + "_cache"].view(-1, hd)[a:a + kv * size].view(kv, size, hd)[:, :ctx[i] + n].double()
                if c["cache"] == "i8":
                    x = x * s[m + "_scale"][a:a + kv * size].view(kv, size, 1)[:, :ctx[i] + n].double()
                return x

            k, v = part("k"), part("v")
            hidden = torch.zeros(n, ctx[i] + n, dtype=torch.bool, device="cuda")
            for t in range(n):
                for u in range(n):
                    if s["mask"] is None:
                        break   # single tokens see themselves
                    hidden[t, ctx[i] + u] = not _bit(s, first + t, u)
        for h in range(c["heads"]):
            score = (s["q"][first:first + n, h].double() @ k[h // group].T.contiguous()) / math.sqrt(hd)
            out[first:first + n, h] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ v[h // group]
        first += n
    return out


def _bit(s, row, u):
    if "mask_host" not in s:
        s["mask_host"] = s["mask"].cpu().numpy().view(np.uint64)
    return bool(int(s["mask_host"][row, u >> 6]) >> (u & 63) & 1)

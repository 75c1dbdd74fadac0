"""Cases of the operators on paged caches and of beam search, which is what moves their pages.

  attend   ss_attention_pages: one new token per row attends to the pages that its row of a page table names.  With beams, rows of one
           group hold the same pages as far as their histories agree.
  store    ss_pages_write, ss_pages_read: keys and values of tokens go to the pages that hold their positions, and are read back.
  select   ss_beam_select: of all continuations of a group's beams the best, by the sum of their tokens' log probabilities (over a power
           of the length), with the beams' histories in their new order.
  fork     ss_pages_fork, ss_pages_copy: rows take over the pages of their parents and grow; pages that nobody holds are handed out, and
           a page that several would write into is copied, in all layers.
  compact  ss_pages_compact, ss_pages_copy: the pages in use move to the lowest numbers.

Widths are those of this repository's models (4 heads of 64; 32 and 40 heads of 128; a vocabulary of 1024 or 32000), and heads that share
4 or 8 key/value heads.  Lengths, histories and parents of a case follow from the case's own numbers (so that `work` can count), whereas the
seed makes the values and, where nothing is counted by it, the places of the pages.

A pool holds pages of `page` slots: element e of head h in slot s of page p is at ((p * kv_heads + h) * page + s) * dim + e; position t of a
row is slot t % page of the page in entry t // page of its table.  In 8 bits a vector is round(x / scale), scale = max|x| / 127.
"""
import functools
import json
import math
import random

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "i8": 1}
BIG = 2**31 - 1


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one row late in a long answer at the 7B widths, cache in 8 bits: the smallest call, all latency
        dict(name="attend_1_long_7b", op="attend", groups=1, beams=1, prompt=3700, tail=200, page=16, heads=32, kv_heads=32, dim=128, type="f16", cache="i8"),
        # a decode step of 64 rows of unlike length with shared heads, cache in 8 bits: bound by the cache's bytes
        dict(name="attend_64_shared", op="attend", groups=64, beams=1, prompt=7600, tail=400, page=64, heads=32, kv_heads=8, dim=128, type="bf16", cache="i8"),
        # beam search, 16 prompts of 8 beams each, which share their prompts' pages and the older part of their answers
        dict(name="attend_16x8_beams", op="attend", groups=16, beams=8, prompt=3001, tail=250, page=16, heads=32, kv_heads=8, dim=128, type="f16", cache="f16"),
        # a decode step of 64 rows: one token each into their last pages
        dict(name="store_step_64", op="store", groups=64, tokens=1, prompt=4000, page=16, kv_heads=8, dim=128, type="bf16", cache="i8"),
        # the keys and values of a prompt forward, a group of prompts at the 7B widths
        dict(name="store_prompts_7b", op="store", groups=128, tokens=180, prompt=0, page=16, kv_heads=32, dim=128, type="f16", cache="i8"),
        # one answer searched with 4 beams, logits as this library's forwards give them
        dict(name="select_1x4", op="select", groups=1, beams=4, keep=4, vocab=32000, width=64, type="f32", power=0.0),
        # a group of prompts with 8 beams each
        dict(name="select_32x8", op="select", groups=32, beams=8, keep=8, vocab=32000, width=512, type="bf16", power=1.0),
        # a large batch over a large vocabulary of odd size
        dict(name="select_96x8_wide", op="select", groups=96, beams=8, keep=8, vocab=100003, width=1024, type="bf16", power=0.6),
        # a beam search's step: 8 prompts of 4 beams change places and grow by a token, four layers' pages are copied
        dict(name="fork_8x4", op="fork", groups=8, beams=4, prompt=1500, tail=200, page=16, layers=4, kv_heads=8, dim=128, cache="f16"),
        # a long step of the same: 64 prompts of 8 beams, 24 layers of shared heads in pages of 64
        dict(name="fork_64x8_deep", op="fork", groups=64, beams=8, prompt=700, tail=300, page=64, layers=24, kv_heads=1, dim=128, cache="f16"),
        # a pool of a small batch that has become sparse
        dict(name="compact_small", op="compact", groups=24, beams=1, prompt=900, tail=100, page=16, spare=0.6, layers=2, kv_heads=4, dim=64, cache="f16"),
        # a large pool, half of it free, 16 layers
        dict(name="compact_large", op="compact", groups=200, beams=2, prompt=2000, tail=300, page=16, spare=1.0, layers=16, kv_heads=1, dim=128, cache="bf16"),
    ]


def draw(rng):
    def upto(lo, hi):   # spread over the logarithm
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(("attend", "attend", "store", "select", "select", "fork", "compact"))
        kv, group = rng.choice(((4, 1), (32, 1), (40, 1), (1, 8), (2, 4), (8, 4), (8, 8), (4, 7)))
        dim, kind = rng.choice((64, 128, 128)), rng.choice(("f16", "bf16"))
        c = dict(op=op)
        if op == "select":
            keep = rng.choice((1, 2, 3, 4, 5, 8, 16))
            c.update(groups=upto(1, 200), beams=rng.choice((1, keep, keep)), keep=keep, vocab=rng.choice((1024, 32000, upto(100, 150000))), width=upto(8, 1024),
                     type=rng.choice(("f32", "f16", "bf16")), power=rng.choice((0.0, 0.6, 1.0)))
        else:
            c.update(groups=upto(1, 200), prompt=upto(1, 20000), page=rng.choice((16, 16, 32, 64, 128, 256)), kv_heads=kv, dim=dim)
            if op == "store":
                c.update(tokens=rng.choice((1, upto(1, 2000))), type=kind, cache=rng.choice(("i8", "i8", kind)))
                c["prompt"] = rng.choice((0, upto(1, 4000)))
            else:
                c.update(beams=rng.choice((1, 1, 2, 3, 4, 8)), tail=upto(1, 400))
            if op == "attend":
                c.update(heads=kv * group, type=kind, cache=rng.choice(("i8", "i8", kind)))
            elif op != "store":
                c.update(layers=upto(1, 24), cache=rng.choice((kind, "i8")))
                if op == "compact":
                    c["spare"] = round(rng.uniform(0.1, 1.5), 2)
        if _size(c) > 2.4e9:
            continue
        w = work(c)
        if w["bytes"] <= 1.2e9 and w["flops"] <= 1e11:
            return c


def _size(c):
    """About how many values the plain form's largest tables hold."""
    if c["op"] == "select":
        return 8 * c["groups"] * c["beams"] * c["vocab"]
    if c["op"] in ("attend", "store"):
        top = c["prompt"] + (c["tokens"] if c["op"] == "store" else c["tail"])
        return c["groups"] * c.get("beams", 1) * top * c["kv_heads"] * c["dim"]
    return 2 * c["groups"] * (c["prompt"] + c["beams"] * (c["tail"] + c["page"])) * (1 + c.get("spare", 0.1)) * c["layers"] * c["kv_heads"] * c["dim"]


# ------------------------------------------------------------------------------------------------ tables of pages
def _lengths(r, n, top, least):
    """n lengths from `least` to `top`, of which one is `top`: without an order, most of them short."""
    got = [least + int((top - least) * r.random() ** 1.5) for _ in range(n)]
    got[r.randrange(n)] = top
    return got


def _book(c):
    return _book_of(json.dumps({k: v for k, v in c.items() if k != "name"}, sort_keys=True))


@functools.lru_cache(maxsize=64)
def _book_of(text):
    """Of a case: the pages of each row (numbered as they were taken), the rows' lengths, how many pages there are."""
    c = json.loads(text)
    r = random.Random(text)
    page, beams, taken = c["page"], c.get("beams", 1), 0
    first = _lengths(r, c["groups"], c["prompt"], min(c["prompt"], 1))
    more = _lengths(r, c["groups"], c["tokens"] if c["op"] == "store" else c["tail"], 1)
    rows, lengths = [], []
    for n, tail in zip(first, more):
        last = []
        for b in range(beams):
            same = n + int(tail * r.random() * 0.8) if b else 0   # a beam agrees with the one before it for the prompt and some of the answer
            pages = last[:same // page]
            while len(pages) * page < n + tail:
                pages.append(taken)
                taken += 1
            rows.append(pages)
            lengths.append(n + tail)
            last = pages
    return rows, lengths, taken, (first, more)


@functools.lru_cache(maxsize=64)
def _parents_of(text):
    """Of a step of beam search: each row's parent in its group, some of them several times; few groups end."""
    c = json.loads(text)
    r = random.Random(text + "parents")
    got = []
    for g in range(c["groups"]):
        ended = r.random() < 0.05
        got += [-1 if ended else g * c["beams"] + min(int(c["beams"] * r.random() ** 2), c["beams"] - 1) for _ in range(c["beams"])]
    return got


def _parents(c):
    return _parents_of(json.dumps({k: v for k, v in c.items() if k != "name"}, sort_keys=True))


def _room(c):
    """Pages of the pool."""
    taken = _book(c)[2]
    if c["op"] == "fork":
        return taken + 2 * len(_book(c)[0]) + 3
    return taken + (int(taken * c["spare"]) + 1 if c["op"] == "compact" else 7)


def _forked(c):
    """Entries that the rows of a fork read and write, and how many pages are copied."""
    rows, lengths, _, _ = _book(c)
    parents, entries, writers, others = _parents(c), 0, {}, set()
    for p in parents:
        if p < 0:
            continue
        entries += len(rows[p]) + -(-(lengths[p] + 1) // c["page"])
        for k, x in enumerate(rows[p]):
            if lengths[p] % c["page"] and k == len(rows[p]) - 1:
                writers[x] = writers.get(x, 0) + 1
            else:
                others.add(x)
    return entries, sum(n - (x not in others) for x, n in writers.items())


def _vector(c):
    return c["dim"] * SIZE[c["cache"]] + (4 if c["cache"] == "i8" else 0)


def work(case):
    c = case
    if c["op"] == "select":   # logits once; states, results and histories are small beside them
        n, m = c["groups"] * c["beams"], c["groups"] * c["keep"]
        return {"bytes": n * (c["vocab"] * SIZE[c["type"]] + 9 + 4 * c["width"]) + m * (17 + 4 * c["width"]), "flops": 4 * n * c["vocab"]}
    rows, lengths, taken, (first, more) = _book(c)
    if c["op"] == "store":   # keys and values come in, lie in their pages, and go out
        n = 2 * sum(more) * c["kv_heads"]
        return {"bytes": n * (4 * c["dim"] + _vector(c)) + 12 * sum(more), "flops": 4 * n * c["dim"]}
    if c["op"] == "attend":   # each page once, as far as some row sees it
        seen = {}
        for pages, n in zip(rows, lengths):
            for k, x in enumerate(pages):
                seen[x] = max(seen.get(x, 0), min(c["page"], n - k * c["page"]))
        entries = sum(len(x) for x in rows)
        return {"bytes": 2 * len(rows) * c["heads"] * c["dim"] * SIZE[c["type"]] + 4 * entries + 2 * sum(seen.values()) * c["kv_heads"] * _vector(c),
                "flops": 4 * sum(lengths) * c["heads"] * c["dim"]}
    block = 4 * c["layers"] * c["page"] * c["kv_heads"] * _vector(c)   # a page's keys and values, read and written
    if c["op"] == "fork":
        entries, copies = _forked(c)
        return {"bytes": 4 * entries + copies * block + 24 * len(rows), "flops": entries}
    entries, n = sum(len(x) for x in rows), _room(c)
    moved = int((_places(c) >= taken).sum())
    return {"bytes": 8 * entries + 4 * n + moved * block, "flops": entries}


def _places(c):
    """Where the pages of a case lie in its pool."""
    return np.random.RandomState(len(_book(c)[0]) + 7 * _book(c)[2]).permutation(_room(c))[:_book(c)[2]]


# ------------------------------------------------------------------------------------------------ inputs
def _vectors(g, n, heads, dim, dtype):
    """Keys, values or queries: normal, with channels of different size, as projections have them."""
    gain = torch.exp(0.4 * torch.randn(heads, dim, device="cuda", generator=g))
    return (torch.randn(n, heads, dim, device="cuda", generator=g) * gain).to(dtype)


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _pool(g, c, n):
    """A layer's pages, full of stored vectors: keys, values, and in 8 bits their scales."""
    got = {}
    for name in ("k", "v"):
        gain = torch.exp(0.4 * torch.randn(c["kv_heads"], 1, c["dim"], device="cuda", generator=g))
        x = torch.randn(n, c["kv_heads"], c["page"], c["dim"], device="cuda", generator=g) * gain
        if c["cache"] == "i8":
            scale = x.abs().amax(-1, keepdim=True) / 127
            got[name], got[name + "_scale"] = torch.round(x / scale).to(torch.int8).reshape(-1), scale.reshape(-1)
        else:
            got[name], got[name + "_scale"] = x.to(TYPES[c["cache"]]).reshape(-1), None
    return got


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "select":
        return _prepare_select(s, c, g, seed)
    rows, lengths, taken, (first, more) = _book(c)
    n = s["n_pages"] = _room(c)
    place = _places(c) if c["op"] == "compact" else np.random.RandomState(seed % 2**32).permutation(n)[:taken]
    stride = max(len(x) for x in rows) + 1 + (c["op"] == "fork")   # room for the next page
    table = np.full((len(rows), stride), -1, np.int32)
    for i, x in enumerate(rows):
        table[i, :len(x)] = place[x]
    s.update(table=_ints(table), lengths=_ints(lengths), stride=stride, max_length=max(lengths))
    if c["op"] == "store":
        s["layer"] = {"k": torch.zeros(n * c["kv_heads"] * c["page"] * c["dim"], dtype=TYPES[c["cache"]], device="cuda"), "k_scale": None}
        if c["cache"] == "i8":
            s["layer"]["k_scale"] = torch.zeros(n * c["kv_heads"] * c["page"], device="cuda")
        s["layer"].update(v=s["layer"]["k"].clone(), v_scale=None if s["layer"]["k_scale"] is None else s["layer"]["k_scale"].clone())
        s["k"], s["v"] = (_vectors(g, sum(more), c["kv_heads"], c["dim"], TYPES[c["type"]]) for _ in range(2))
        s["row"] = _ints(np.repeat(np.arange(len(rows)), more).tolist())
        s["pos"] = _ints(np.concatenate([a + np.arange(b) for a, b in zip(first, more)]).tolist())
        return s
    if c["op"] == "attend":
        s["layer"] = _pool(g, c, n)
        s["q"] = _vectors(g, len(rows), c["heads"], c["dim"], TYPES[c["type"]])
        return s
    s["layers"] = [_pool(g, c, n) for _ in range(c["layers"])]
    s["new_table"], s["new_lengths"] = torch.full_like(s["table"], -1), torch.zeros_like(s["lengths"])
    if c["op"] == "fork":
        s["parent"] = _ints(_parents(c))
    return s


def _prepare_select(s, c, g, seed):
    """Logits as models give them: a few tokens far above the rest, some forbidden ones; sums of beams that have come some way, best first."""
    r = random.Random(seed)
    rows, vocab = c["groups"] * c["beams"], c["vocab"]
    x = torch.randn(rows, vocab, device="cuda", generator=g) * 2
    some = 40
    likely = (torch.randint(vocab, (rows, 1), device="cuda", generator=g) + torch.arange(some, device="cuda") * (vocab // some)) % vocab   # no token twice
    x.scatter_(1, likely, 8 + 3 * torch.randn(rows, some, device="cuda", generator=g))
    x[:, torch.randint(vocab, (vocab // 50,), device="cuda", generator=g)] = -math.inf
    s["end_id"] = r.randrange(vocab)
    x[:, s["end_id"]] = 6 + 3 * torch.randn(rows, device="cuda", generator=g)
    s["logits"] = x.to(TYPES[c["type"]])
    totals = -torch.rand(c["groups"], c["beams"], device="cuda", generator=g).cumsum(1) * 4 - 20 * torch.rand(c["groups"], 1, device="cuda", generator=g)
    s["totals"] = totals.contiguous()
    steps = torch.randint(1, c["width"], (c["groups"], 1), device="cuda", generator=g)
    ended = torch.rand(c["groups"], c["beams"], device="cuda", generator=g) < 0.15
    back = (torch.rand(c["groups"], c["beams"], device="cuda", generator=g) * steps).long()
    length = torch.where(ended, (steps - back).clamp_min(1), steps)
    s["ended"], s["lengths"] = ended.to(torch.uint8).view(-1), length.to(torch.int32).view(-1)
    history = torch.randint(vocab, (rows, c["width"]), device="cuda", generator=g)
    s["history"] = history.masked_fill(torch.arange(c["width"], device="cuda") >= length.view(-1, 1), -1).to(torch.int32)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c)
    return {"attend": _plain_attend, "store": _plain_store, "select": _plain_select, "fork": _plain_fork, "compact": _plain_compact}[c["op"]](s, c)


def _own(s, c):
    from paper_2305_13144_amd import binding as ss

    if c["op"] == "select":
        return tuple(ss.ss_beam_select(s["logits"], s["totals"], c["keep"], lengths=s["lengths"], ended=s["ended"], end_id=s["end_id"],
                                       length_power=c["power"], history=s["history"]))
    if "handle" not in s:   # what a program keeps with its pool: views of the tensors, nothing computed
        s["handle"] = [ss.Pages(x["k"], x["v"], c["page"], c["kv_heads"], c["dim"], x["k_scale"], x["v_scale"]) for x in s.get("layers") or [s["layer"]]]
        s["rows"] = ss.PageTable(s["table"], s["lengths"], c["page"], s["n_pages"])
        if "new_table" in s:
            s["new_rows"] = ss.PageTable(s["new_table"], s["new_lengths"], c["page"], s["n_pages"])
    layers, rows = s["handle"], s["rows"]
    if c["op"] == "attend":
        return ss.ss_attention_pages(s["q"], layers[0], rows, s["max_length"], group=c["beams"])
    if c["op"] == "store":
        if c["tokens"] == 1:   # the decode step: a token a row, at its end
            ss.ss_pages_write(layers[0], rows, s["k"], s["v"])
            return ss.ss_pages_read(layers[0], rows, dtype=s["k"].dtype)
        ss.ss_pages_write(layers[0], rows, s["k"], s["v"], s["row"], s["pos"])
        return ss.ss_pages_read(layers[0], rows, s["row"], s["pos"], s["k"].dtype)
    if c["op"] == "fork":
        src, dst, missing = ss.ss_pages_fork(rows, s["new_rows"], s["parent"])
        ss.ss_pages_copy(layers, src, dst)
        return s["new_table"], s["new_lengths"], src, dst, missing, _tensors(s)
    src, dst, place, counts = ss.ss_pages_compact(rows, s["new_rows"])
    ss.ss_pages_copy(layers, src, dst, counts[1:])
    return s["new_table"], s["new_lengths"], src, dst, place, counts, _tensors(s)


def _tensors(s):
    """The first and last layer: the others are copied alike."""
    return [x for layer in (s["layers"][0], s["layers"][-1]) for x in layer.values() if x is not None]


def _vector_of(s, c, row, pos):
    """Number of the vector of each head at the given positions: [..., heads]."""
    page = s["table"][row.long(), (pos // c["page"]).long()].long().unsqueeze(-1)
    return (page * c["kv_heads"] + torch.arange(c["kv_heads"], device="cuda")) * c["page"] + (pos % c["page"]).long().unsqueeze(-1)


def _held(s, c, name, at):
    x = s["layer"][name].view(-1, c["dim"])[at].float()
    return x * s["layer"][name + "_scale"][at].unsqueeze(-1) if c["cache"] == "i8" else x


def _plain_store(s, c):
    at = _vector_of(s, c, s["row"], s["pos"])

    def write(name):
        x = s[name].float()
        if c["cache"] == "i8":
            scale = x.abs().amax(-1) / 127
            x = torch.where(scale.unsqueeze(-1) > 0, torch.round(x / scale.unsqueeze(-1)), 0.0)
            s["layer"][name + "_scale"][at] = scale
        s["layer"][name].view(-1, c["dim"])[at] = x.to(TYPES[c["cache"]])
        return _held(s, c, name, at).to(s[name].dtype)

    return write("k"), write("v")


def _plain_attend(s, c):
    n, top, kv, hd = len(s["lengths"]), s["max_length"], c["kv_heads"], c["dim"]
    group = c["heads"] // kv
    length = s["lengths"].unsqueeze(-1)
    pos = torch.minimum(torch.arange(top, device="cuda").expand(n, top), length - 1)
    at = _vector_of(s, c, torch.arange(n, device="cuda").unsqueeze(-1).expand(n, top), pos).transpose(1, 2)   # [n, kv, top]
    q = s["q"].float().view(n, kv, group, hd)
    scores = torch.matmul(q, _held(s, c, "k", at).transpose(2, 3).contiguous()) * hd ** -0.5
    scores = scores.masked_fill((torch.arange(top, device="cuda") >= length).view(n, 1, 1, top), -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    out = torch.matmul(p, _held(s, c, "v", at)) / p.sum(-1, keepdim=True)
    return out.reshape(n, c["heads"], hd).to(s["q"].dtype)


def _plain_select(s, c):
    groups, beams, keep, vocab = c["groups"], c["beams"], c["keep"], c["vocab"]
    x = s["logits"].double()
    real = torch.isfinite(x)
    top = x.masked_fill(~real, -math.inf).amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).masked_fill(~real, 0.0).sum(-1, keepdim=True))
    total, length, ended = s["totals"].double().view(-1, 1), s["lengths"].double().view(-1, 1), s["ended"].bool().view(-1, 1)
    new = total + (x - lse)
    rank = new / (length + 1) ** c["power"]
    rank = rank.masked_fill(~real | ended | ~torch.isfinite(total), -math.inf)
    stay = torch.where(ended & torch.isfinite(total), total / length.clamp_min(1) ** c["power"], -math.inf)   # an ended beam as it is
    end = s["end_id"]
    rank[:, end] = torch.where(ended.view(-1), stay.view(-1), rank[:, end])
    new[:, end] = torch.where(ended.view(-1), total.view(-1), new[:, end])
    rank, new = rank.view(groups, beams * vocab), new.view(groups, beams * vocab)
    picked, every = [], torch.arange(beams * vocab, device="cuda")
    for _ in range(keep):   # the largest, of several the first
        best = rank.amax(-1, keepdim=True)
        at = torch.where((rank == best) & (best > -math.inf), every, beams * vocab).amin(-1, keepdim=True)
        picked.append(at)
        rank.scatter_(1, at.clamp_max(beams * vocab - 1), -math.inf)
    at = torch.cat(picked, 1)
    there = at < beams * vocab
    at = at.clamp_max(beams * vocab - 1)
    row = (torch.arange(groups, device="cuda").unsqueeze(-1) * beams + at // vocab).view(-1)
    there, token = there.view(-1), (at % vocab).view(-1)
    sums = torch.where(there, new.gather(1, at).view(-1), -math.inf).float().view(groups, keep)
    old, over = s["lengths"].long()[row], s["ended"].bool()[row]
    length = torch.where(there, old + ~over, 0)
    slot = torch.arange(c["width"], device="cuda")
    kept = torch.where((slot < old.unsqueeze(-1)), s["history"][row], -1)
    kept = torch.where((slot == old.unsqueeze(-1)) & ~over.unsqueeze(-1), token.int().unsqueeze(-1), kept)
    kept = torch.where(there.unsqueeze(-1), kept, -1)
    return (torch.where(there, row, -1).int(), torch.where(there, token, -1).int(), sums, length.int(), (~there | over | (token == end)).to(torch.uint8), kept)


def _plain_copy(s, src, dst):
    there = src >= 0
    a, b = src[there].long(), dst[there].long()
    for layer in s["layers"]:
        for x in layer.values():
            if x is not None:
                x.view(s["n_pages"], -1)[b] = x.view(s["n_pages"], -1)[a]


def _plain_fork(s, c):
    page, n, stride = c["page"], s["n_pages"], s["stride"]
    parent = s["parent"].long()
    has, i = parent >= 0, torch.arange(len(parent), device="cuda")
    old = torch.where(has, s["lengths"].long()[parent.clamp_min(0)], 0)
    new = torch.where(has, (old + 1).clamp_max(stride * page), 0)
    held, wanted = (old + page - 1) // page, (new + page - 1) // page
    entry = torch.arange(stride, device="cuda")
    table = torch.where(entry < held.unsqueeze(-1), s["table"].long()[parent.clamp_min(0)], -1)
    writes = (old % page > 0) & (new > old)
    last = (held - 1).clamp_min(0)
    # of each page the lowest row that writes into it, -1 if one holds it that does not, BIG if none does
    claim = torch.where(writes.unsqueeze(-1) & (entry == last.unsqueeze(-1)), i.unsqueeze(-1), -1)
    owner = torch.full((n + 1,), BIG, device="cuda", dtype=torch.int64)
    owner.scatter_reduce_(0, torch.where(table >= 0, table, n).view(-1), claim.reshape(-1), "amin")
    owner = owner[:n]
    source = table.gather(1, last.unsqueeze(-1)).view(-1)
    copies = writes & (owner[source.clamp_min(0)] != i)
    need = wanted - held + copies.long()
    start = need.cumsum(0) - need
    free = torch.cat([torch.nonzero(owner == BIG).view(-1), torch.full((int(need.sum()),), -1, device="cuda")])
    missing = (need.sum() - (owner == BIG).sum()).clamp_min(0)
    dst = torch.where(copies, free[start], -1)
    table.scatter_(1, last.unsqueeze(-1), torch.where(copies, dst, source).unsqueeze(-1))
    more = (entry >= held.unsqueeze(-1)) & (entry < wanted.unsqueeze(-1))
    rank = (start + copies.long()).unsqueeze(-1) + entry - held.unsqueeze(-1)
    table = torch.where(more, free[torch.where(more, rank, 0)], table)
    src = torch.where(dst >= 0, source, -1)
    s["new_table"].copy_(torch.where(has.unsqueeze(-1), table, -1))
    s["new_lengths"].copy_(new)
    _plain_copy(s, src, dst)
    return s["new_table"], s["new_lengths"], src.int(), dst.int(), missing.int().view(1), _tensors(s)


def _plain_compact(s, c):
    n, page = s["n_pages"], c["page"]
    there = torch.arange(s["stride"], device="cuda") < ((s["lengths"] + page - 1) // page).unsqueeze(-1)
    used = torch.zeros(n, dtype=torch.bool, device="cuda")
    used[s["table"][there].long()] = True
    count = int(used.sum())
    holes, high = torch.nonzero(~used[:count]).view(-1), torch.nonzero(used[count:]).view(-1) + count
    place = torch.where(used, torch.arange(n, device="cuda"), -1)
    place[high] = holes
    src, dst = (torch.full((n // 2,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    src[:len(high)], dst[:len(high)] = high.int(), holes.int()
    s["new_table"].copy_(torch.where(there, place[s["table"].long().clamp_min(0)], -1))
    s["new_lengths"].copy_(s["lengths"])
    _plain_copy(s, src, dst)
    return s["new_table"], s["new_lengths"], src, dst, place.int(), _ints([count, len(high)]), _tensors(s)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    """Attention, what 8 bits hold, and the sums of beams; what is whole numbers or copied has no such value."""
    c = case
    if c["op"] in ("fork", "compact"):
        return None
    s = prepare(c, seed)
    if c["op"] == "store":
        def stored(x):
            x = x.double()
            if c["cache"] != "i8":
                return x
            unit = x.abs().max(dim=2, keepdim=True).values / 127
            return torch.where(unit > 0, (x / unit).round() * unit, x)
        return stored(s["k"]), stored(s["v"])
    if c["op"] == "select":
        return _exact_select(s, c)
    hd, kv, page = c["dim"], c["kv_heads"], c["page"]
    out = torch.empty(len(s["lengths"]), kv, c["heads"] // kv, hd, dtype=torch.float64, device="cuda")
    table, lengths = s["table"].cpu().numpy(), s["lengths"].tolist()
    for i, n in enumerate(lengths):
        pages = torch.tensor(table[i, :-(-n // page)].astype(np.int64), device="cuda")

        def part(m):   # [kv, n, dim]
            x = s["layer"][m].view(-1, kv, page, hd)[pages].double()
            if c["cache"] == "i8":
                x = x * s["layer"][m + "_scale"].view(-1, kv, page, 1)[pages].double()
            return x.permute(1, 0, 2, 3).reshape(kv, -1, hd)[:, :n]

        score = s["q"][i].double().view(kv, -1, hd) @ part("k").transpose(1, 2).contiguous() / math.sqrt(hd)
        out[i] = torch.softmax(score, -1) @ part("v").contiguous()
    return out.view(len(lengths), c["heads"], hd)


def _exact_select(s, c):
    beams, keep, vocab, end = c["beams"], c["keep"], c["vocab"], s["end_id"]
    totals, lengths, ended = s["totals"].view(-1).tolist(), s["lengths"].tolist(), s["ended"].tolist()
    sums = torch.full((c["groups"], keep), -math.inf, dtype=torch.float64, device="cuda")
    for g in range(c["groups"]):
        rank, total = [], []
        for b in range(beams):
            r = g * beams + b
            x = s["logits"][r].double()
            x = torch.where(torch.isfinite(x), x, -math.inf)
            if ended[r]:
                t = torch.full((vocab,), -math.inf, dtype=torch.float64, device="cuda")
                t[end] = totals[r]
            else:
                t = totals[r] + (x - torch.logsumexp(x, 0))
            total.append(t)
            rank.append(t / max(lengths[r] + (not ended[r]), 1) ** c["power"])
        rank, total = torch.cat(rank), torch.cat(total)
        n = min(keep, len(rank))
        order = torch.sort(rank, descending=True, stable=True).indices[:n]
        sums[g, :n] = total[order]
    return None, None, sums, None, None, None

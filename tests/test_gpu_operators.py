"""The operators on device tensors against their definitions in 64 bits: caches in 8 and 16 bits, attention of single tokens and
of drafted trees over them, causal attention of packed prompts, at the sizes, masks, strides and values where they can go
wrong, and a run of them together.

Tolerance of an attention result.  With weights w_s = p_s / sum p, A = sum w_s |v_s| and half a step eps / 2 of the type that a
value is rounded to, relative to the value (2^-11 for half, 2^-8 for bf16):
  the result itself                       eps/2 |out|
  the weights, as operands (half or the 16-bit cache's type)      eps_w/2 A, and below half's normal range 2^-25 of the largest weight, for
                                          each slot: n 2^-23 max|v| covers both it and the scales' power of two
  the scores, sums of dim products in fp32 and the exponential    each weight by at most 4 D relative, D = (dim + 8) 2^-24 scale max sum|q||k|
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2305_13144_amd import binding as ss

pytestmark = pytest.mark.gpu

F16, BF16, I8 = torch.float16, torch.bfloat16, torch.int8


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def assert_attention(got, q, k, v, visible, scale, weight_type):
    """got, q [rows, dim]; k, v [slots, dim] in 64 bits; visible [rows, slots]."""
    q64, n = q.double(), k.shape[0]
    s = (q64 @ k.T.contiguous()) * scale
    s = s.masked_fill(~visible, -math.inf)
    top = s.max(-1, keepdim=True).values if n else torch.zeros(len(q), 1, device=q.device, dtype=torch.float64)
    p = torch.where(visible, torch.exp(s - top.clamp_min(-1e300)), 0.0)
    total = p.sum(-1, keepdim=True)
    w = torch.where(total > 0, p / total.clamp_min(1e-300), 0.0)
    ref, A = w @ v, w @ v.abs()
    D = (q.shape[1] + 8) * 2.0 ** -24 * abs(scale) * (q64.abs() @ k.abs().T.contiguous()).masked_fill(~visible, 0).amax(-1, keepdim=True)
    vmax = torch.where(visible.any(0, keepdim=True).T, v.abs(), 0.0).max() if n else 0.0
    tol = half_step(got.dtype) * ref.abs() + (half_step(weight_type) + 4 * D + 2.0 ** -18) * A + n * 2.0 ** -23 * vmax + 1e-30
    bad = (got.double() - ref).abs() > tol
    assert torch.isfinite(got).all()
    assert not bad.any(), (bad.sum().item(), (got.double() - ref).abs().max().item(), tol[bad].min().item())


class Held:
    """A cache of random vectors in every slot, with slabs in no order, and what it stands for in 64 bits."""

    def __init__(self, seed, slots, kv, dim, dtype, scale_spread=0.0):
        g = gen(seed)
        total, order = sum(slots), np.random.default_rng(seed).permutation(len(slots))
        start, at = np.zeros(len(slots), np.int64), 0
        for i in order:
            start[i], at = at, at + slots[i]
        self.start, self.slots, self.kv, self.dim = start, slots, kv, dim
        parts = {}
        for name in ("k", "v"):
            x = randn(g, total * kv, dim)
            if dtype == I8:
                x = x * torch.exp(scale_spread * randn(g, total * kv, 1))
                unit = x.abs().amax(-1) / 127
                parts[name] = torch.round(x / unit[:, None]).to(I8)
                parts[name + "_scale"] = unit
            else:
                parts[name] = x.to(dtype)
        self.raw = parts
        self.cache = ss.Cache(parts["k"].reshape(-1), parts["v"].reshape(-1), torch.tensor(start, device="cuda"), i32(slots), kv, dim,
                              parts.get("k_scale"), parts.get("v_scale"))

    def rows(self, name, seq, head, n):
        a = int(self.start[seq]) * self.kv + head * self.slots[seq]
        x = self.raw[name][a:a + n].double()
        return x * self.raw[name + "_scale"][a:a + n, None].double() if name + "_scale" in self.raw else x


# ------------------------------------------------------------------------------------------------ write and read
def codes_of(x):
    """Scale and codes as defined, with numpy's float32 divisions (rounded to nearest)."""
    x = x.float().cpu().numpy()
    unit = np.abs(x).max(-1) / np.float32(127)
    with np.errstate(all="ignore"):
        c = np.where(unit[..., None] > 0, np.rint(x / unit[..., None]), 0)
    return unit, np.clip(c, -127, 127).astype(np.int8)


@pytest.mark.parametrize("n", [1, 3, 67])
@pytest.mark.parametrize("kv,dim", [(1, 64), (4, 64), (8, 128), (5, 128)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("held", [I8, F16, BF16])
def test_tokens_are_held_and_read_back_as_defined(n, kv, dim, dtype, held):
    g = gen(n)
    slots = [9, 0, 40, 33]
    c = ss.Cache.allocate(slots, kv, dim, held)
    for x in (c.k, c.v):
        x.fill_(3)
    wide = randn(g, n, 3 * kv + 2, dim, dtype=dtype)             # keys and values are views of a wider projection
    k, v = wide[:, 1:1 + kv], wide[:, 2 + kv:2 + 2 * kv]
    places = [(i, s) for i in range(4) for s in range(slots[i])]
    pick = np.random.default_rng(n).permutation(len(places))[:n]
    seq, slot = [places[i][0] for i in pick], [places[i][1] for i in pick]
    if n > 2:                                                    # tokens that do not exist: padding, past the slab, no such sequence
        seq[0], slot[1] = -1, 40
        if n > 60:
            seq[50], slot[60], seq[61], slot[62] = 4, -1, 1, 2**30
    here = [t for t in range(n) if 0 <= seq[t] < 4 and 0 <= slot[t] < slots[seq[t]]]
    ss.ss_cache_write(c, k, v, i32(seq), i32(slot))
    rk, rv = (torch.full((n, kv, dim), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    ss.ss_cache_read(c, i32(seq), i32(slot), k=rk, v=rv)
    start = np.cumsum([0] + slots)
    for x, r, store, unit in ((k, rk, c.k, c.k_scale), (v, rv, c.v, c.v_scale)):
        want = torch.full_like(store, 3).view(-1, dim)
        at = torch.tensor([[start[seq[t]] * kv + h * slots[seq[t]] + slot[t] for h in range(kv)] for t in here], device="cuda").view(len(here), kv)
        if held == I8:
            scale, codes = codes_of(x)
            want[at] = torch.tensor(codes, device="cuda")[here]
            assert torch.equal(unit[at].cpu(), torch.tensor(scale)[here])
            value = (torch.tensor(codes).float() * torch.tensor(scale)[..., None]).to(dtype)
        else:
            want[at] = x[here].to(held)
            value = x.to(held).to(dtype).cpu()
        assert torch.equal(store.view(-1, dim), want)            # the rest of the cache is as it was
        back = torch.full((n, kv, dim), 7.0, dtype=dtype)
        back[here] = value[here]
        assert torch.equal(r.cpu(), back)                        # and so are rows of tokens that do not exist


@pytest.mark.parametrize("dim", [64, 128])
def test_every_quotient_gets_the_nearest_code(dim):
    """Vectors whose elements lie at, and one step around, the middles between codes, over sizes from subnormal to huge; one error
    in a thousand quotients that are near a middle would show."""
    r = np.random.default_rng(5)
    n = 512
    top = np.exp2(r.uniform(-120, 120, (n, 1, 1))).astype(np.float32)
    top[:8] = np.float32(2.0) ** np.array([-133, -132, -130, -127, -126, -101, -100, -99], np.float32).reshape(8, 1, 1)
    x = top / np.float32(127) * (r.integers(-127, 127, (n, 3, dim)) + np.float32(0.5)).astype(np.float32)
    x = torch.tensor(x).to(BF16)
    near = x.view(torch.int16) + torch.tensor(r.integers(-1, 2, x.shape).astype(np.int16))
    x = near.view(BF16)
    x[..., 0] = torch.tensor(top[:, :, 0]).to(BF16)
    x = x.cuda()
    c = ss.Cache.allocate([n], 3, dim, I8)
    ss.ss_cache_write(c, x, x, i32([0] * n), i32(list(range(n))))
    scale, codes = codes_of(x)
    assert np.array_equal(c.k.view(3, n, dim).cpu().numpy(), codes.transpose(1, 0, 2))
    assert np.array_equal(c.v_scale.view(3, n).cpu().numpy(), scale.T, equal_nan=True)   # a step below zero is a NaN


def test_zeros_and_infinities_and_nan():
    x = torch.ones(6, 1, 128, dtype=F16, device="cuda")
    x[0] = 0
    x[1, 0, 5] = math.inf
    x[2, 0, 127] = math.nan
    x[3] = 6e-8
    x[4] = -65504
    c = ss.Cache.allocate([6], 1, 128, I8)
    at = i32(range(6))
    ss.ss_cache_write(c, x, x, i32([0] * 6), at)
    k, v = ss.ss_cache_read(c, i32([0] * 6), at, F16)
    assert torch.equal(k[0], x[0]) and torch.equal(k[3:], x[3:])
    assert k[1].isnan().all() and v[2].isnan().all()
    assert torch.equal(k[0], v[0]) and torch.equal(k[3:], v[3:])
    h = ss.Cache.allocate([6], 1, 128, F16)
    big = torch.tensor([1e9, -1e9, math.inf, math.nan], dtype=BF16, device="cuda").repeat(32).view(1, 1, 128)
    ss.ss_cache_write(h, big, big, i32([0]), i32([2]))
    got = h.k.view(6, 128)[2, :4].cpu()
    assert got[:3].tolist() == [65504, -65504, 65504] and got[3].isnan()


# ------------------------------------------------------------------------------------------------ attention over a cache
def random_tree(r, n):
    return [int(r.integers(-1, t)) if t else -1 for t in range(n)]


def check_tree(seed, ctx, nodes, kv, group, dim, dtype, held, chain=False, spread=0.0, max_context=None, empty_rows=False, scale=None):
    r = np.random.default_rng(seed)
    heads, n = kv * group, len(ctx)
    slots = [a + b + int(r.integers(0, 9)) for a, b in zip(ctx, nodes)]
    H = Held(seed, slots, kv, dim, held, spread)
    first = np.concatenate([[0], np.cumsum(nodes)])
    rows, top = int(first[-1]) + 3, max(max(nodes), 1)
    big = randn(gen(seed + 1), rows, heads + 2, dim, dtype=dtype)
    q = big[:, 1:1 + heads]
    out = torch.full((rows, heads, dim), 5.0, dtype=dtype, device="cuda")
    mask = None
    bits = np.zeros((rows, top), bool)
    if not chain:
        words = (top + 63) // 64
        packed = np.zeros((rows, words), np.int64)
        for i in range(n):
            m = ss.ss_tree_mask(random_tree(r, nodes[i]), top)
            packed[first[i]:first[i + 1]] = m
        if empty_rows:
            packed[r.random(rows) < 0.5] = 0
        bits = (packed.view(np.uint64)[:, np.arange(top) // 64] >> (np.arange(top) % 64).astype(np.uint64) & np.uint64(1)).astype(bool)
        mask = torch.tensor(packed, device="cuda")
    got = ss.ss_attention_tree(q, H.cache, i32(ctx), max(ctx) if max_context is None else max_context, nodes=i32(first.tolist()),
                               max_nodes=top, mask=mask, out=out, scale=scale)
    assert got is out
    assert (out[first[-1]:] == 5).all()
    for i in range(n):
        if nodes[i] == 0:
            continue
        see = np.ones((nodes[i], ctx[i] + nodes[i]), bool)
        see[:, ctx[i]:] = np.tril(np.ones((nodes[i], nodes[i]), bool)) if chain else bits[first[i]:first[i + 1], :nodes[i]]
        see = torch.tensor(see, device="cuda")
        for h in range(heads):
            k, v = (H.rows(m, i, h // group, ctx[i] + nodes[i]) for m in ("k", "v"))
            assert_attention(out[first[i]:first[i + 1], h], q[first[i]:first[i + 1], h], k, v, see, dim ** -0.5 if scale is None else scale,
                             F16 if held == I8 else held)
    return H, q, out


HELD = [(F16, F16), (BF16, BF16), (F16, I8), (BF16, I8)]


@pytest.mark.parametrize("dtype,held", HELD)
@pytest.mark.parametrize("kv,group,dim", [(4, 1, 64), (2, 1, 128), (1, 8, 128), (2, 7, 64), (1, 20, 128)])
def test_single_tokens(dtype, held, kv, group, dim):
    ctx = [0, 1, 31, 32, 33, 127, 128, 129, 500, 1025]
    check_tree(1, ctx, [1] * len(ctx), kv, group, dim, dtype, held, chain=True)


@pytest.mark.parametrize("dtype,held", HELD)
@pytest.mark.parametrize("kv,group,dim", [(3, 1, 128), (2, 4, 128), (1, 7, 64)])
@pytest.mark.parametrize("chain", [False, True])
def test_trees(dtype, held, kv, group, dim, chain):
    check_tree(2, [0, 5, 64, 300, 0, 1000], [1, 17, 0, 33, 61, 8], kv, group, dim, dtype, held, chain=chain)


@pytest.mark.parametrize("dtype,held", HELD)
def test_more_nodes_than_a_word_of_the_mask_has_bits(dtype, held):
    check_tree(3, [10, 0, 700], [64, 65, 200], 1, 2, 128, dtype, held)


@pytest.mark.parametrize("dtype,held", HELD)
def test_rows_that_see_nothing_are_zero(dtype, held):
    H, q, out = check_tree(4, [0, 3, 0], [40, 7, 1], 2, 3, 64, dtype, held, empty_rows=True)
    assert (out[:40] == 0).all(-1).all(-1).any()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_scales_of_very_different_size(dtype):
    check_tree(5, [700, 90], [9, 1], 2, 2, 128, dtype, I8, spread=6.0)


@pytest.mark.parametrize("held", [F16, I8])
@pytest.mark.parametrize("said", [0, 100, 2**30])
def test_the_stated_context_only_shares_out_the_work(held, said):
    check_tree(6, [3000, 20], [5, 2], 1, 2, 128, F16, held, max_context=said)


@pytest.mark.parametrize("dtype,held", HELD)
def test_a_long_context_is_shared_out_and_joined(dtype, held):
    check_tree(7, [20000, 11, 4097], [3, 1, 20], 1, 4, 128, dtype, held)


@pytest.mark.parametrize("dtype,held", HELD)
@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0])
def test_scales_of_scores(dtype, held, scale):
    check_tree(60, [130, 0], [3, 1], 2, 2, 128, dtype, held, scale=scale)
    check_tree(61, [40, 0], [20, 30], 1, 4, 64, dtype, held, scale=scale)
    if held != I8:
        check_packed(62, [40, 200], 1, 2, 64, dtype, scale=scale)


@pytest.mark.parametrize("dtype,most", [(F16, 65504.0), (BF16, math.inf)])
@pytest.mark.parametrize("nodes", [1, 40])
def test_infinite_values_reach_those_who_see_them(nodes, dtype, most):
    """A value that is infinite makes that element of those who see it infinite (half: its largest number), with its sign, and no other."""
    H = Held(63, [100], 1, 128, dtype)
    q = randn(gen(64), nodes, 1, 128, dtype=dtype)
    call = lambda: ss.ss_attention_tree(q, H.cache, i32([50]), 50, nodes=i32([0, nodes]), max_nodes=nodes)  # noqa: E731
    clean = call()
    H.raw["v"][50 + nodes - 1, 5], H.raw["v"][50 + nodes - 1, 77] = math.inf, -math.inf
    got = call()
    assert got[-1, 0, 5] == most and got[-1, 0, 77] == -most
    got[-1, 0, [5, 77]] = clean[-1, 0, [5, 77]]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype,most", [(F16, 65504.0), (BF16, math.inf)])
def test_infinite_values_in_prompts(dtype, most):
    """As above; of both signs they make a NaN of what sees both, wherever in the prompt they are."""
    k, v, q = (randn(gen(s), 300, 1, 128, dtype=dtype) for s in (65, 66, 67))
    call = lambda: ss.ss_attention_packed(q, k, v, i32([0, 300]), 300)  # noqa: E731
    clean = call()
    v[266, 0, 3] = -math.inf
    v[5, 0, 70], v[270, 0, 70] = math.inf, -math.inf
    got = call()
    assert (got[266:, 0, 3] == -most).all() and (got[5:270, 0, 70] == most).all() and got[270:, 0, 70].isnan().all()
    got[266:, 0, 3], got[5:, 0, 70] = clean[266:, 0, 3], clean[5:, 0, 70]
    assert torch.equal(got, clean)


def test_results_by_heads_and_inputs_that_all_share():
    """Results as [heads][rows], and one row of queries for all nodes."""
    H = Held(68, [60, 60], 2, 64, I8)
    one = randn(gen(69), 1, 4, 64, dtype=BF16)
    out = torch.empty(4, 2, 64, dtype=BF16, device="cuda").transpose(0, 1)
    ss.ss_attention_tree(one.expand(2, 4, 64), H.cache, i32([30, 50]), 50, out=out)
    want = ss.ss_attention_tree(one.repeat(2, 1, 1), H.cache, i32([30, 50]), 50)
    assert torch.equal(out, want)
    assert torch.equal(ss.ss_attention_tree(one.expand(2, 4, 64), H.cache, i32([30, 50]), 50, stream=0), want)


@pytest.mark.parametrize("nodes,context", [(1, 200), (1, 5000), (20, 200), (100, 3000)])
@pytest.mark.parametrize("held", [F16, I8])
def test_results_in_the_place_of_the_queries(held, nodes, context):
    H = Held(72, [context + nodes] * 3, 2, 128, held)
    q, table = randn(gen(73), 3 * nodes, 8, 128, dtype=F16), i32([0, nodes, 2 * nodes, 3 * nodes])
    call = lambda q, out: ss.ss_attention_tree(q, H.cache, i32([context, context // 2, 0]), context, nodes=table, max_nodes=nodes, out=out)  # noqa: E731
    want, own = call(q, None), q.clone()
    assert call(own, own) is own and torch.equal(own, want)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_results_of_prompts_in_the_place_of_the_queries(dtype):
    q, k, v = randn(gen(74), 700, 8, 64, dtype=dtype), randn(gen(75), 700, 2, 64, dtype=dtype), randn(gen(76), 700, 2, 64, dtype=dtype)
    offsets = i32([0, 1, 130, 700])
    want, own = ss.ss_attention_packed(q, k, v, offsets, 570), q.clone()
    assert ss.ss_attention_packed(own, k, v, offsets, 64 * 65535, out=own) is own and torch.equal(own, want)


@pytest.mark.parametrize("dtype,held", HELD)
def test_many_small_weights_count_beside_a_large_one(dtype, held):
    """One slot of score 0 and thousands whose weights, 2^-15 each, are below half's normal range: together a quarter."""
    n, dim = 8192, 128
    k = torch.zeros(n, 1, dim, device="cuda")
    k[:, 0, 0] = -1
    k[77, 0, 0] = 0
    v = randn(gen(70), n, 1, dim) + 1
    H = Held(71, [n], 1, dim, held)
    H.raw["k"].copy_(k[:, 0])
    if held == I8:
        H.raw["k_scale"].fill_(1)
    else:
        H.raw["v"].copy_(v[:, 0])
    q = torch.zeros(1, 1, dim, dtype=dtype, device="cuda")
    q[0, 0, 0] = 15
    out = ss.ss_attention_tree(q, H.cache, i32([n - 1]), n, scale=math.log(2))
    kk, vv = H.rows("k", 0, 0, n), H.rows("v", 0, 0, n)
    assert_attention(out[:, 0], q[:, 0], kk, vv, torch.ones(1, n, dtype=torch.bool, device="cuda"), math.log(2), F16 if held == I8 else held)
    if held != I8:
        qs = torch.zeros(n, 1, dim, dtype=dtype, device="cuda")
        qs[-1] = q[0]
        out = ss.ss_attention_packed(qs, k.to(dtype), v.to(dtype), i32([0, n]), n, scale=math.log(2))
        assert_attention(out[-1:, 0], q[:, 0], kk, vv, torch.ones(1, n, dtype=torch.bool, device="cuda"), math.log(2), dtype)


def test_the_same_call_gives_the_same_bits():
    H, q, out = check_tree(8, [5000, 40], [7, 30], 2, 4, 128, BF16, I8)
    ctx, nodes = i32([5000, 40]), i32([0, 7, 37])
    a, b = (ss.ss_attention_tree(q, H.cache, ctx, 5000, nodes=nodes, max_nodes=30)[:37] for _ in range(2))
    assert torch.equal(a, b)


@pytest.mark.parametrize("held", [F16, BF16, I8])
def test_unseen_slots_have_no_influence_whatever_they_hold(held):
    """Slots behind the nodes, and nodes that a row does not see, hold infinities and NaN."""
    dtype = BF16 if held == BF16 else F16
    ctx, nodes, kv, group, dim = [50, 0], [20, 3], 2, 2, 128
    H = Held(9, [90, 40], kv, dim, held)
    q = randn(gen(10), 23, kv * group, dim, dtype=dtype)
    parents = [random_tree(np.random.default_rng(9), 20), [-1, -1, 1]]
    mask = torch.tensor(np.concatenate([ss.ss_tree_mask(p, 20) for p in parents]), device="cuda")
    call = lambda: ss.ss_attention_tree(q, H.cache, i32(ctx), 50, nodes=i32([0, 20, 23]), max_nodes=20, mask=mask)  # noqa: E731
    clean = call()
    for i, hidden in ((0, 7), (1, 0)):
        a = [int(H.start[i]) * kv + h * H.slots[i] for h in range(kv)]
        for name, junk in (("k", math.nan), ("v", math.inf)):
            for first in a:
                x = H.raw[name + "_scale"] if held == I8 else H.raw[name]
                x[first + ctx[i] + hidden] = junk
                x[first + ctx[i] + nodes[i]:first + H.slots[i]] = junk
    got = call()
    sees = (mask.cpu().numpy()[:, 0] >> np.where(np.arange(23) < 20, 7, 0) & 1).astype(bool)
    assert sees.any() and not sees.all()
    sees = torch.tensor(sees, device="cuda")
    assert torch.isnan(got[sees]).any(-1).all()
    assert torch.isfinite(got[~sees]).all()
    assert (got[~sees].float() - clean[~sees].float()).abs().max() <= 2.0 ** -7 * clean.float().abs().max()   # a bf16 step of other sums


def test_sequences_are_chosen_and_missing_ones_give_zeros():
    H = Held(11, [30, 50, 20], 2, 64, I8)
    q = randn(gen(12), 5, 4, 64, dtype=F16)
    seq, ctx = [2, 0, 7, -1, 2], [19, 4, 3, 3, 100]              # a sequence twice; none; a context beyond its slab
    out = ss.ss_attention_tree(q, H.cache, i32(ctx), 100, seq=i32(seq))
    assert (out[2:4] == 0).all()
    for j, n in ((0, 20), (1, 5), (4, 20)):
        for h in range(4):
            k, v = (H.rows(m, seq[j], h // 2, n) for m in ("k", "v"))
            assert_attention(out[j:j + 1, h], q[j:j + 1, h], k, v, torch.ones(1, n, dtype=torch.bool, device="cuda"), 0.125, F16)


def test_tables_that_lead_outside_are_not_followed():
    """Slabs beyond the cache, node tables beyond the rows: nothing is read or written there, the others are as always."""
    H = Held(13, [30, 50], 1, 128, F16)
    bad = ss.Cache(H.cache.k, H.cache.v, torch.tensor([0, 70], device="cuda"), i32([30, 50]), 1, 128)   # the cache has 80 slots
    q = randn(gen(14), 2, 1, 128, dtype=F16)
    out = ss.ss_attention_tree(q, bad, i32([9, 9]), 9)
    assert (out[1] == 0).all() and (out[0] != 0).any()
    k = torch.ones(2, 1, 128, dtype=F16, device="cuda")
    before = H.cache.k.clone()
    ss.ss_cache_write(bad, k, k, i32([1, 1]), i32([9, 0]))
    assert torch.equal(before, H.cache.k)
    out = torch.full_like(q, 5.0)
    ss.ss_attention_tree(q, H.cache, i32([9, 9]), 9, nodes=i32([-1, 1, 3]), max_nodes=3, out=out)
    assert (out == 5).all()


def test_a_cache_beyond_two_to_the_32_elements():
    kv, dim, far = 8, 128, 4_300_000                              # 4.4e9 elements each
    k8 = torch.zeros((far + 300) * kv * dim, dtype=I8, device="cuda")
    scale = torch.zeros((far + 300) * kv, device="cuda")
    c = ss.Cache(k8, k8.clone(), torch.tensor([0, far], device="cuda"), i32([far, 300]), kv, dim, scale, scale.clone())
    g = gen(15)
    k, v = (randn(g, 200, kv, dim, dtype=F16) for _ in range(2))
    seq, slot = i32([1] * 150 + [0] * 50), i32(list(range(150)) + list(range(far - 50, far)))
    ss.ss_cache_write(c, k, v, seq, slot)
    rk, rv = ss.ss_cache_read(c, seq, slot, F16)
    for x, r in ((k, rk), (v, rv)):
        assert ((x.float() - r.float()).abs() <= x.float().abs().amax(-1, keepdim=True) * (0.5 / 127 + 2.0 ** -10)).all()
    q = randn(g, 1, kv, dim, dtype=F16)
    out = ss.ss_attention_tree(q, c, i32([149]), 149, seq=i32([1]))
    units = [torch.tensor(codes_of(x)[0], device="cuda") for x in (k, v)]
    codes = [torch.tensor(codes_of(x)[1], device="cuda") for x in (k, v)]
    for h in range(kv):
        kk, vv = (a[:150, h].double() * u[:150, h, None].double() for a, u in zip(codes, units))
        assert_attention(out[:, h], q[:, h], kk, vv, torch.ones(1, 150, dtype=torch.bool, device="cuda"), dim ** -0.5, F16)


# ------------------------------------------------------------------------------------------------ packed prompts
def check_packed(seed, lens, kv, group, dim, dtype, scale=None, gain=1.0):
    heads, first = kv * group, np.concatenate([[0], np.cumsum(lens)])
    rows = int(first[-1]) + 5
    wide = gain * randn(gen(seed), rows, heads + 2 * kv, dim)
    wide = wide.to(dtype)
    q, k, v = wide[:, :heads], wide[:, heads:heads + kv], wide[:, heads + kv:]
    wide[first[-1]:] = math.nan                                   # rows behind the last sequence
    out = torch.full((rows, heads, dim), 5.0, dtype=dtype, device="cuda")
    ss.ss_attention_packed(q, k, v, i32(first.tolist()), max(lens), scale=scale, out=out)
    assert (out[first[-1]:] == 5).all()
    for i, n in enumerate(lens):
        part = slice(int(first[i]), int(first[i + 1]))
        see = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        for h in range(heads):
            if n:
                assert_attention(out[part, h], q[part, h], k[part, h // group].double(), v[part, h // group].double(), see,
                                 dim ** -0.5 if scale is None else scale, dtype)
    return q, k, v, out


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("kv,group,dim", [(4, 1, 64), (2, 1, 128), (1, 4, 128), (2, 7, 64)])
@pytest.mark.parametrize("lens", [[1], [1, 0, 2, 15, 16, 17, 33], [63, 64, 65, 127, 128, 129, 0], [255, 256, 257, 3], [600, 1, 385]])
def test_packed_prompts(dtype, kv, group, dim, lens):
    check_packed(20, lens, kv, group, dim, dtype)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_packed_prompts_with_peaked_and_flat_weights(dtype):
    check_packed(21, [300, 70], 1, 2, 128, dtype, gain=3.0)
    check_packed(22, [300, 70], 1, 2, 128, dtype, scale=0.0)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_long_packed_prompt(dtype):
    check_packed(23, [2500], 1, 2, 128, dtype)


@pytest.mark.parametrize("n", [40, 300, 700])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dim", [64, 128])
def test_later_tokens_have_no_influence_whatever_they_hold(n, dtype, dim):
    q, k, v, clean = check_packed(24, [n, n], 1, 2, dim, dtype)
    k, v, at = k.clone(), v.clone(), n - 9
    k[at:n], v[at:n] = math.nan, math.inf
    v[n + at:2 * n], k[n + at] = math.nan, math.inf
    got = ss.ss_attention_packed(q, k, v, i32([0, n, 2 * n]), n)
    for a in (0, n):
        assert torch.isfinite(got[a:a + at]).all()
        assert (got[a:a + at].float() - clean[a:a + at].float()).abs().max() <= 2.0 ** -7 * clean[:2 * n].float().abs().max()
        assert not torch.isfinite(got[a + at:a + n]).any()


def test_what_lies_beyond_the_stated_length_is_passed_over():
    q, k, v, out = check_packed(25, [90, 30], 2, 1, 64, F16)
    part = torch.full_like(out, 5.0)
    ss.ss_attention_packed(q, k, v, i32([0, 90, 120]), 50, out=part)
    assert torch.equal(part[:50], out[:50]) and torch.equal(part[90:120], out[90:120]) and (part[50:90] == 5).all()
    part.fill_(5)
    ss.ss_attention_packed(q, k, v, i32([-1, 90, 500]), 90, out=part)      # tables that lead outside
    assert (part == 5).all()


# ------------------------------------------------------------------------------------------------ calls
def test_calls_of_nothing():
    c = ss.Cache.allocate([4], 2, 64, I8)
    none = torch.empty(0, 2, 64, dtype=F16, device="cuda")
    ss.ss_cache_write(c, none, none, i32([]), i32([]))
    ss.ss_cache_read(c, i32([]), i32([]), F16)
    assert ss.ss_attention_tree(none, c, i32([]), 0).shape == (0, 2, 64)
    assert ss.ss_attention_packed(none, none, none, i32([0]), 0).shape == (0, 2, 64)
    empty = ss.Cache.allocate([], 2, 64, F16)
    k = torch.ones(1, 2, 64, dtype=F16, device="cuda")
    ss.ss_cache_write(empty, k, k, i32([0]), i32([0]))


def test_a_whole_answer_on_another_stream_and_in_a_graph():
    """Prompts, their cache, and drafted chains behind them: the drafts' results are those of the whole sequences as prompts, in
    eager calls, on a stream of their own, and in a graph that is replayed after other work on new inputs."""
    kv, group, dim, dtype = 2, 4, 128, BF16
    lens, extra = [70, 1, 200], [5, 3, 9]
    whole = [a + b for a, b in zip(lens, extra)]
    off = np.concatenate([[0], np.cumsum(whole)])
    old = np.concatenate([np.arange(off[i], off[i] + lens[i]) for i in range(3)])
    new = np.concatenate([np.arange(off[i] + lens[i], off[i + 1]) for i in range(3)])
    seq = np.repeat(np.arange(3), whole)
    slot = np.concatenate([np.arange(n) for n in whole])
    at = {name: i32(x.tolist()) for name, x in dict(seq_old=seq[old], slot_old=slot[old], seq_new=seq[new], slot_new=slot[new], off=off,
                                                   old_off=np.concatenate([[0], np.cumsum(lens)]), nodes=np.concatenate([[0], np.cumsum(extra)])).items()}
    old, new = torch.tensor(old, device="cuda"), torch.tensor(new, device="cuda")
    mask = torch.tensor(np.concatenate([ss.ss_tree_mask(list(range(-1, n - 1)), 9) for n in extra]), device="cuda")
    q, k, v = (torch.empty(int(off[-1]), h, dim, dtype=dtype, device="cuda") for h in (kv * group, kv, kv))
    c16, c8 = ss.Cache.allocate(whole, kv, dim, dtype), ss.Cache.allocate(whole, kv, dim, I8)

    def steps(stream=None):
        res = [ss.ss_attention_packed(q[old], k[old], v[old], at["old_off"], max(lens), stream=stream)]
        for c in (c16, c8):
            ss.ss_cache_write(c, k[old], v[old], at["seq_old"], at["slot_old"], stream=stream)
            ss.ss_cache_write(c, k[new], v[new], at["seq_new"], at["slot_new"], stream=stream)
            res.append(ss.ss_attention_tree(q[new], c, i32_lens, 200, nodes=at["nodes"], max_nodes=9, mask=mask, stream=stream))
        return res

    i32_lens = i32(lens)

    def fill(seed):
        for x, s in ((q, 0), (k, 1), (v, 2)):
            x.copy_(randn(gen(seed + s), *x.shape, dtype=dtype))

    fill(30)
    eager = steps()
    full = ss.ss_attention_packed(q, k, v, at["off"], max(whole))
    assert torch.equal(eager[0], full[old])
    scale = full.float().abs().max()
    assert (eager[1].float() - full[new].float()).abs().max() <= 2 * 2.0 ** -8 * scale       # two roundings to bf16, and the weights'
    # codes off by half a step: a value by max|v| / 254, a score by about sqrt(dim) max|q| max|k| / 254 / sqrt(dim), at most 0.1 here
    assert (eager[2].float() - full[new].float()).abs().max() <= (0.25 + 2.0 ** -7) * v.float().abs().max()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = steps()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, again))
    raw = steps(stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, raw))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = steps()
    for seed in (40, 50, 60):
        fill(seed)
        want = [x.clone() for x in steps()]
        for c in (c16, c8):
            c.k.zero_()
            c.v.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, captured)), seed


# ------------------------------------------------------------------------------------------------ large scores
def check_best_slot(got, q, k, v, visible, scale, weight=0.0):
    """Where the best score leads by more than what fp32 sums of products leave open, the result is that slot's value (one rounding of
    the result; with 16 bits a weight and its sum are the same number).  Returns how many rows are decided so.
    weight: with 8 bits the result is half(p scale / R) R code / p, by the one rounding to half within 2^-11 of scale code."""
    s = ((q.double() @ k.T.contiguous()) * scale).masked_fill(~visible, -math.inf)
    best = s.topk(2, -1)
    open_ = 4 * (q.shape[1] + 8) * 2.0 ** -24 * abs(scale) * (q.double().abs() @ k.abs().T.contiguous()).masked_fill(~visible, 0).amax(-1)
    sure = best.values[:, 0] - best.values[:, 1] > open_ + 60                              # 2^-86: no other slot has a weight
    want = v[best.indices[:, 0]]
    assert torch.isfinite(got).all()
    assert ((got.double() - want).abs() <= (half_step(got.dtype) + weight) * want.abs())[sure].all()
    return int(sure.sum())


@pytest.mark.parametrize("dtype,size", [(F16, 1e4), (BF16, 1e6), (BF16, 1e15), (BF16, 2e18)])
@pytest.mark.parametrize("scale", [1.0, -1.0])
@pytest.mark.parametrize("nodes,context", [(1, 60), (3, 400), (9, 70), (20, 900)])
def test_large_scores(nodes, context, scale, dtype, size):
    """Scores from 2^30 on, whose steps in fp32 are larger than the exponential's range."""
    group, dim = 3, 128
    H = Held(84, [context + nodes], 1, dim, dtype)
    H.raw["k"].copy_((H.raw["k"].double() * size).to(dtype))
    q = (randn(gen(85), nodes, group, dim).double() * size).to(dtype)
    got = ss.ss_attention_tree(q, H.cache, i32([context]), context, nodes=i32([0, nodes]), max_nodes=nodes, scale=scale)
    k, v = (H.rows(m, 0, 0, context + nodes) for m in ("k", "v"))
    see = torch.ones(nodes, context + nodes, dtype=torch.bool, device="cuda").tril(context)
    assert sum(check_best_slot(got[:, h], q[:, h], k, v, see, scale) for h in range(group)) >= nodes * group // 2


@pytest.mark.parametrize("dtype,size", [(F16, 1e4), (BF16, 1e6), (BF16, 1e15), (BF16, 2e18)])
@pytest.mark.parametrize("scale", [1.0, -1.0])
@pytest.mark.parametrize("dim", [64, 128])
def test_large_scores_in_prompts(dim, scale, dtype, size):
    n = 300
    q, k = ((randn(gen(s), n, 1, dim).double() * size).to(dtype) for s in (86, 87))
    v = randn(gen(88), n, 1, dim, dtype=dtype)
    got = ss.ss_attention_packed(q, k, v, i32([0, n]), n, scale=scale)
    see = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    assert check_best_slot(got[:, 0], q[:, 0], k[:, 0].double(), v[:, 0].double(), see, scale) >= n // 2


# ------------------------------------------------------------------------------------------------ rows and slots of very different size
@pytest.mark.parametrize("dtype,held", HELD)
@pytest.mark.parametrize("nodes,kv,group,dim,context", [(4, 2, 4, 128, 40), (8, 1, 4, 64, 300), (40, 1, 8, 128, 90), (33, 2, 1, 64, 700), (8, 1, 2, 128, 6000)])
def test_rows_have_nothing_to_do_with_their_neighbours(nodes, kv, group, dim, context, dtype, held):
    """Queries that are infinite, no numbers, huge or tiny beside ordinary ones (other nodes, and other heads of the same node): each row
    is what it is by its own definition.  A huge row's answer is the value of its best slot."""
    heads, big = kv * group, 1e30 if dtype == BF16 else 6e4
    H = Held(80, [context + nodes], kv, dim, held)
    q = randn(gen(81), nodes, heads, dim, dtype=dtype)
    odd = {(0, 0): "inf", (1, heads - 1): "nan", (2, 0): "huge", (nodes - 1, heads - 1): "tiny"}
    q[0, 0, 3], q[1, heads - 1, dim - 1] = -math.inf, math.nan
    q[2, 0] = (q[2, 0].double() * big / 8).to(dtype)
    q[nodes - 1, heads - 1] = (q[nodes - 1, heads - 1].double() * (1e-30 if dtype == BF16 else 1e-3)).to(dtype)
    got = ss.ss_attention_tree(q, H.cache, i32([context]), context, nodes=i32([0, nodes]), max_nodes=nodes)
    see = torch.ones(nodes, context + nodes, dtype=torch.bool, device="cuda").tril(context)
    for h in range(heads):
        k, v = (H.rows(m, 0, h // group, context + nodes) for m in ("k", "v"))
        plain = torch.tensor([odd.get((t, h)) in (None, "tiny") for t in range(nodes)], device="cuda")
        assert_attention(got[plain, h], q[plain, h], k, v, see[plain], dim ** -0.5, F16 if held == I8 else held)
        for t in range(nodes):
            if odd.get((t, h)) in ("inf", "nan"):
                assert got[t, h].isnan().all()
            elif odd.get((t, h)) == "huge":
                s = torch.where(see[t], k @ q[t, h].double(), -math.inf)
                best = s.topk(2)
                if (best.values[0] - best.values[1]) * dim ** -0.5 > 2.0 ** -12 * (k.abs() @ q[t, h].double().abs()).max() + 60:   # no other slot has a weight
                    want = v[best.indices[0]]
                    assert ((got[t, h].double() - want).abs() <= (half_step(dtype) + 2.0 ** -10) * want.abs()).all()


@pytest.mark.parametrize("dtype,held", HELD)
@pytest.mark.parametrize("nodes,group", [(12, 1), (30, 1), (150, 2)])
def test_large_queries_that_see_little(nodes, group, dtype, held):
    """Queries of 2^13 and more whose rows see nothing, their last node alone, or a node of the last steps: what they do not see comes first."""
    H = Held(89, [nodes], 1, 128, held)
    q = (randn(gen(90), nodes, group, 128) * 2.0 ** (20 if dtype == BF16 else 12)).to(dtype)
    bits = torch.zeros(nodes, nodes, dtype=torch.bool)
    bits[1::3, nodes - 1] = True
    bits[2::3, nodes - 2:] = True
    words = (nodes + 63) // 64
    mask = torch.tensor([[sum(int(b) << i for i, b in enumerate(row[64 * w:64 * w + 64])) for w in range(words)] for row in bits.tolist()], device="cuda")
    got = ss.ss_attention_tree(q, H.cache, i32([0]), 0, nodes=i32([0, nodes]), max_nodes=nodes, mask=mask)
    assert (got[0::3] == 0).all()
    v = H.rows("v", 0, 0, nodes)
    assert ((got[1::3].double() - v[-1]).abs() <= (half_step(dtype) + 2.0 ** -11) * v[-1].abs()).all()   # one slot: its weight is rounded, 8 bits
    k, see = H.rows("k", 0, 0, nodes), bits.cuda()
    for h in range(group):
        check_best_slot(got[2::3, h], q[2::3, h], k, v, see[2::3], 128 ** -0.5, 2.0 ** -11 if held == I8 else 0.0)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("nodes,group", [(1, 1), (5, 4), (60, 2)])
@pytest.mark.parametrize("far", [0, 12, 20, 40, 100])
def test_a_slot_of_large_values_and_no_weight(nodes, group, far, dtype):
    """One slot whose values are 2^far times the others' and whose weight is 2^-far / 16 or less: the others count as without it.

    Tolerance, A and D as above: per slot a rounding to half of weight times scale, relative 2^-11 above half's normal range, below it
    2^-25 in units of which the largest product that the row met is at least 2^6: over n slots n 2^-31 of that product times 127."""
    dim, context = 128, 200
    H = Held(82, [context + nodes], 1, dim, I8)
    k, unit = H.raw["k"], H.raw["k_scale"]
    first = int(H.start[0])
    k[:, 0] = 0                                     # the first element of a key is the far slot's alone
    k[first + 70] = 0
    k[first + 70, 0] = -127
    unit[first + 70] = 1
    H.raw["v_scale"][first + 70] *= 2.0 ** far
    q = randn(gen(83), nodes, group, dim, dtype=dtype)
    q[..., 0] = (far + 4 + 12) * math.log(2) * dim ** 0.5 / 127   # 12: the others' scores lie well above -12 in powers of two
    got = ss.ss_attention_tree(q, H.cache, i32([context]), context, nodes=i32([0, nodes]), max_nodes=nodes)
    kk, vv = (H.rows(m, 0, 0, context + nodes) for m in ("k", "v"))
    see = torch.ones(nodes, context + nodes, dtype=torch.bool, device="cuda").tril(context)
    scale = H.raw["v_scale"][first:first + context + nodes].double()
    for h in range(group):
        q64 = q[:, h].double()
        s = ((q64 @ kk.T.contiguous()) * dim ** -0.5).masked_fill(~see, -math.inf)
        w = torch.softmax(s, -1)
        assert (w[:, 70] * 2.0 ** far <= 1 / 16).all()
        ref, A = w @ vv, w @ vv.abs()
        D = (dim + 8) * 2.0 ** -24 * dim ** -0.5 * (q64.abs() @ kk.abs().T.contiguous()).masked_fill(~see, 0).amax(-1, keepdim=True)
        tol = half_step(dtype) * ref.abs() + (half_step(F16) + 4 * D + 2.0 ** -18) * A + kk.shape[0] * 2.0 ** -31 * 127 * (w * scale).amax(-1, keepdim=True)
        bad = (got[:, h].double() - ref).abs() > tol
        assert not bad.any(), (bad.sum().item(), (got[:, h].double() - ref).abs().max().item())


# ------------------------------------------------------------------------------------------------ streams
def busy():
    """Some milliseconds of work on the current stream."""
    a = torch.ones(4096, 4096, device="cuda")
    for _ in range(20):
        a = a @ a * 2.0 ** -12
    return a


def calls_on(stream, H, x, tables):
    """Every operator, its inputs and tables made by the current stream just before, nothing of them kept."""
    q, k, v = x.clone(), x[:, :2].clone(), x[:, 2:4].clone()
    seq, slot, context, nodes = (lambda a=a: a.clone() for a in tables)
    ss.ss_cache_write(H.cache, k, v, seq(), slot(), stream=stream)
    res = list(ss.ss_cache_read(H.cache, seq(), slot(), F16, stream=stream))
    res.append(ss.ss_attention_tree(q, H.cache, context(), 40, nodes=nodes(), max_nodes=3, stream=stream))
    res.append(ss.ss_attention_packed(x.clone(), k.clone(), v.clone(), nodes(), 3, stream=stream))
    return res


def held_calls(seed):
    H, x = Held(seed, [60, 60], 2, 128, I8), randn(gen(seed + 1), 4, 8, 128, dtype=F16)
    tables = i32([0, 0, 0, 1]), i32([40, 41, 42, 5]), i32([40, 5]), i32([0, 3, 4])
    return H, x, tables, calls_on(None, H, x, tables), torch.cuda.Stream()


def test_a_given_stream_waits_for_what_the_current_one_holds():
    H, x, tables, want, side = held_calls(91)
    torch.cuda.synchronize()
    late = torch.zeros_like(x)
    busy()
    late.copy_(x)
    got = calls_on(side.cuda_stream, H, late, tables)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_given_stream_keeps_the_memory_that_it_reads():
    H, x, tables, want, side = held_calls(93)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy()                                                    # side reads late
    got = calls_on(side.cuda_stream, H, x, tables)
    junk = [torch.full((n,), 1000, dtype=torch.int16, device="cuda") for n in (x.numel(), x.numel() // 4, 256, 8, 4, 2) for _ in range(12)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(junk) == 72


def test_a_given_stream_in_a_captured_graph():
    """A branch of a captured graph, on the stream given; and the stream itself being captured."""
    H, x, side = Held(95, [60, 60], 2, 128, I8), randn(gen(96), 4, 8, 128, dtype=F16), torch.cuda.Stream()
    call = lambda stream: ss.ss_attention_tree(x, H.cache, i32_40, 40, stream=stream)  # noqa: E731
    i32_40, graph = i32([40, 5]), torch.cuda.CUDAGraph()
    x = x[:2]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        a = call(side.cuda_stream)
        torch.cuda.current_stream().wait_stream(side)
        b = call(torch.cuda.current_stream().cuda_stream)
    for seed in (97, 98, 99):
        x.copy_(randn(gen(seed), *x.shape, dtype=F16))
        want = call(None).clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, want)


def test_inputs_that_require_gradients_are_refused():
    """A result without a gradient would pass for a constant.  Without gradients the call is as always."""
    H, x, tables, want, side = held_calls(100)
    x = x.requires_grad_()
    seq, slot, context, nodes = tables
    k = x[:, :2]
    for call in (lambda: ss.ss_cache_write(H.cache, k, k.detach(), seq, slot), lambda: ss.ss_cache_write(H.cache, k.detach(), k, seq, slot),
                 lambda: ss.ss_attention_tree(x, H.cache, context, 40, nodes=nodes, max_nodes=3),
                 lambda: ss.ss_attention_tree(x.detach(), H.cache, context, 40, nodes=nodes, max_nodes=3, out=torch.zeros_like(x).requires_grad_()),
                 lambda: ss.ss_attention_packed(x.detach(), k.detach(), k, nodes, 3), lambda: ss.ss_attention_packed(x, k.detach(), k.detach(), nodes, 3)):
        with pytest.raises(ValueError, match="gradients"):
            call()
    with torch.no_grad():
        got = calls_on(None, H, x, tables)
    assert all(torch.equal(a, b) and not a.requires_grad for a, b in zip(got, want))


def test_an_error_that_others_left_behind_is_not_the_calls():
    """A device that does not exist is refused by the runtime, which remembers it; the operators' launches are in order all the same."""
    with open("/proc/self/maps") as f:
        runtime = ctypes.CDLL(next(line.split()[-1] for line in f if "libamdhip64" in line))
    H, x, tables, want, side = held_calls(102)
    seq, slot, context, nodes = tables
    for call in (lambda: ss.ss_cache_write(H.cache, x[:, :2], x[:, 2:4], seq, slot), lambda: ss.ss_cache_read(H.cache, seq, slot, k=x[:, :2], v=x[:, 2:4]),
                 lambda: ss.ss_attention_tree(x, H.cache, context, 40, nodes=nodes, max_nodes=3),
                 lambda: ss.ss_attention_packed(x, x[:, :2], x[:, 2:4], nodes, 3)):
        torch.cuda.synchronize()
        assert runtime.hipSetDevice(100000) != 0
        call()


def test_numbers_beyond_32_bits_are_refused():
    H, x, tables, want, side = held_calls(104)
    seq, slot, context, nodes = tables
    for big in (2**32 + 3, 2**31):
        with pytest.raises(ValueError, match="max_context"):
            ss.ss_attention_tree(x, H.cache, context, big, nodes=nodes, max_nodes=3)
        with pytest.raises(ValueError, match="max_nodes"):
            ss.ss_attention_tree(x, H.cache, context, 40, nodes=nodes, max_nodes=big)
        with pytest.raises(ValueError, match="max_len"):
            ss.ss_attention_packed(x, x[:, :2], x[:, 2:4], nodes, big)


# ------------------------------------------------------------------------------------------------ every slot once, and no more than the roundings
def assert_roundings(got, q, k, v, visible, scale, held, unit=None):
    """As assert_attention, with the roundings of each weight alone.  Weights w of sum 1, the largest w_max:
      16 bits of bf16   each w by 2^-8 of itself
      half              each by 2^-11 of itself or, where it is a subnormal, by 2^-25 of a unit that is no larger than w_max, and never by
                        more than itself: sum over slots min(w, 2^-25 w_max) |v|
      8 bits            each w scale by 2^-11 of itself or 2^-25 R with 2^6 R at most the largest w scale: sum min(w |v|, 2^-31 127 max(w scale))
    unit: the values' scales [slots], with 8 bits."""
    q64 = q.double()
    s = ((q64 @ k.T.contiguous()) * scale).masked_fill(~visible, -math.inf)
    w = torch.softmax(s, -1)
    ref, A = w @ v, w @ v.abs()
    D = (q.shape[1] + 8) * 2.0 ** -24 * abs(scale) * (q64.abs() @ k.abs().T.contiguous()).masked_fill(~visible, 0).amax(-1, keepdim=True)
    small = torch.zeros_like(ref)
    if held == F16:
        small = torch.minimum(w, 2.0 ** -25 * w.amax(-1, keepdim=True)) @ v.abs()
    elif held == I8:
        most = 2.0 ** -31 * 127 * (w * unit).amax(-1)
        small = torch.stack([torch.minimum(row[:, None] * v.abs(), m).sum(0) for row, m in zip(w, most)])
    tol = half_step(got.dtype) * ref.abs() + (half_step(BF16 if held == BF16 else F16) + 4 * D + 2.0 ** -18) * A + small
    bad = (got.double() - ref).abs() > tol
    assert torch.isfinite(got).all()
    assert not bad.any(), (bad.sum().item(), ((got.double() - ref).abs() / tol).max().item())


@pytest.mark.parametrize("dtype,held", HELD)
@pytest.mark.parametrize("nodes,group", [([1, 1, 1], 1), ([3, 1, 2], 4), ([6, 1, 8], 4), ([17, 1, 20], 4)])
def test_long_contexts_to_the_roundings(nodes, group, dtype, held):
    ctx, dim = [20000, 11, 4097], 128
    H = Held(106, [a + b + 3 for a, b in zip(ctx, nodes)], 1, dim, held)
    first = np.concatenate([[0], np.cumsum(nodes)])
    q = randn(gen(107), int(first[-1]), group, dim, dtype=dtype)
    got = ss.ss_attention_tree(q, H.cache, i32(ctx), max(ctx), nodes=i32(first.tolist()), max_nodes=max(nodes))
    for i, n in enumerate(nodes):
        k, v = (H.rows(m, i, 0, ctx[i] + n) for m in ("k", "v"))
        at = int(H.start[i])
        unit = H.raw["v_scale"][at:at + ctx[i] + n].double() if held == I8 else None
        see = torch.ones(n, ctx[i] + n, dtype=torch.bool, device="cuda").tril(ctx[i])
        for h in range(group):
            assert_roundings(got[first[i]:first[i + 1], h], q[first[i]:first[i + 1], h], k, v, see, dim ** -0.5, held, unit)


@pytest.mark.parametrize("dtype,held", HELD)
@pytest.mark.parametrize("nodes,group", [([1], 4), ([4, 1], 4), ([8, 2], 4), ([20], 4), ([33, 1, 70], 1)])
@pytest.mark.parametrize("said", [None, 0, 100000])
def test_every_slot_counts_once(nodes, group, said, dtype, held):
    """Equal weights, and values that say to which of 128 runs of neighbouring slots a slot belongs: a result is the share of the run among
    what the row sees, which one slot too few or too many changes by 1 / (slots of a run) of itself, 1/56 and more here."""
    dim, n = 128, len(nodes)
    ctx = [7000, 130, 1999][:n]
    slots = [a + b for a, b in zip(ctx, nodes)]
    H = Held(108, slots, 1, dim, held)
    for i in range(n):
        run = -(-slots[i] // 128)
        ones = torch.nn.functional.one_hot(torch.arange(slots[i], device="cuda") // run, dim)
        H.raw["v"][int(H.start[i]):int(H.start[i]) + slots[i]] = (ones * (127 if held == I8 else 1)).to(held)
    if held == I8:
        H.raw["v_scale"].fill_(0.5)
    first = np.concatenate([[0], np.cumsum(nodes)])
    q = randn(gen(109), int(first[-1]), group, dim, dtype=dtype)
    got = ss.ss_attention_tree(q, H.cache, i32(ctx), max(ctx) if said is None else said, nodes=i32(first.tolist()), max_nodes=max(nodes), scale=0.0)
    for i in range(n):
        v = H.rows("v", i, 0, slots[i])
        for t in range(nodes[i]):
            want = v[:ctx[i] + t + 1].sum(0) / (ctx[i] + t + 1)       # weights of 1 and halves of powers of two are exact in half
            assert ((got[first[i] + t].double() - want).abs() <= (half_step(dtype) + 2.0 ** -20) * want).all(), (i, t)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dim", [64, 128])
def test_every_token_of_a_prompt_counts_once(dim, dtype):
    lens, heads = [2500, 1, 129, 640], 2
    first = np.concatenate([[0], np.cumsum(lens)])
    q, k = randn(gen(110), int(first[-1]), heads, dim, dtype=dtype), randn(gen(111), int(first[-1]), 1, dim, dtype=dtype)
    v = torch.cat([torch.nn.functional.one_hot(torch.arange(n, device="cuda") // -(-n // dim), dim) for n in lens])[:, None]
    got = ss.ss_attention_packed(q, k, v.to(dtype), i32(first.tolist()), max(lens), scale=0.0)
    for i, n in enumerate(lens):
        seen = v[first[i]:first[i + 1], 0].double().cumsum(0) / torch.arange(1, n + 1, device="cuda")[:, None]
        assert ((got[first[i]:first[i + 1]].double() - seen[:, None]).abs() <= (half_step(dtype) + 2.0 ** -20) * seen[:, None]).all(), i


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_prompts_written_in_8_bits_and_attended(dtype):
    """Prompts into the cache, drafts behind them, and their attention, to the roundings of what the cache then stands for."""
    kv, group, dim, lens, extra = 2, 4, 128, [70, 1, 200], [5, 3, 9]
    whole = [a + b for a, b in zip(lens, extra)]
    c, first = ss.Cache.allocate(whole, kv, dim, I8), np.concatenate([[0], np.cumsum(extra)])
    for part, base in ((lens, [0, 0, 0]), (extra, lens)):
        k, v = (randn(gen(112 + sum(part) + i), sum(part), kv, dim, dtype=dtype) for i in range(2))
        ss.ss_cache_write(c, k, v, i32(np.repeat(np.arange(3), part).tolist()), i32(np.concatenate([b + np.arange(n) for b, n in zip(base, part)]).tolist()))
    q = randn(gen(120), sum(extra), kv * group, dim, dtype=dtype)
    got = ss.ss_attention_tree(q, c, i32(lens), max(lens), nodes=i32(first.tolist()), max_nodes=max(extra))
    start = np.concatenate([[0], np.cumsum(whole)])
    for i in range(3):
        see = torch.ones(extra[i], whole[i], dtype=torch.bool, device="cuda").tril(lens[i])
        for h in range(kv * group):
            at = int(start[i]) * kv + h // group * whole[i]
            units = [x[at:at + whole[i]].double() for x in (c.k_scale, c.v_scale)]
            k, v = (x.view(-1, dim)[at:at + whole[i]].double() * u[:, None] for x, u in zip((c.k, c.v), units))
            assert_roundings(got[first[i]:first[i + 1], h], q[first[i]:first[i + 1], h], k, v, see, dim ** -0.5, I8, units[1])


@pytest.mark.parametrize("held", [BF16, I8])
@pytest.mark.parametrize("nodes,group", [(2, 2), (20, 1), (40, 3)])
@pytest.mark.parametrize("power", [-116, -100, -60, 60, 100, 116])
def test_queries_and_keys_whose_sizes_cancel(nodes, group, power, held):
    """Queries times 2^power, keys times 2^-power: ordinary scores, at both ends of bf16's range."""
    dim, context = 128, 150
    H = Held(121, [context + nodes], 1, dim, held)
    q = randn(gen(122), nodes, group, dim, dtype=BF16)
    call = lambda q: ss.ss_attention_tree(q, H.cache, i32([context]), context, nodes=i32([0, nodes]), max_nodes=nodes)  # noqa: E731
    see = torch.ones(nodes, context + nodes, dtype=torch.bool, device="cuda").tril(context)
    if held == I8:
        H.raw["k_scale"].mul_(2.0 ** -power)
        unit = H.raw["v_scale"].double()
    else:
        H.raw["k"].mul_(2.0 ** -power)
        unit = None
    q = (q.double() * 2.0 ** power).to(BF16)
    got = call(q)
    k, v = (H.rows(m, 0, 0, context + nodes) for m in ("k", "v"))
    for h in range(group):
        assert_roundings(got[:, h], q[:, h], k, v, see, dim ** -0.5, held, unit)


@pytest.mark.parametrize("dtype,size", [(F16, 1e4), (BF16, 1e6), (BF16, 1e15), (BF16, 2e18)])
@pytest.mark.parametrize("scale", [1.0, -1.0])
@pytest.mark.parametrize("nodes,context", [(1, 60), (3, 400), (9, 70), (20, 900)])
def test_large_scores_over_8_bits(nodes, context, scale, dtype, size):
    """As test_large_scores."""
    group, dim = 3, 128
    H = Held(123, [context + nodes], 1, dim, I8)
    H.raw["k_scale"].mul_(size)
    q = (randn(gen(124), nodes, group, dim).double() * size).to(dtype)
    got = ss.ss_attention_tree(q, H.cache, i32([context]), context, nodes=i32([0, nodes]), max_nodes=nodes, scale=scale)
    k, v = (H.rows(m, 0, 0, context + nodes) for m in ("k", "v"))
    see = torch.ones(nodes, context + nodes, dtype=torch.bool, device="cuda").tril(context)
    assert sum(check_best_slot(got[:, h], q[:, h], k, v, see, scale, 2.0 ** -11) for h in range(group)) >= nodes * group // 2


def test_tensors_of_other_dimensions_are_refused():
    H, x, tables, want, side = held_calls(125)
    seq, slot, context, nodes = tables
    k = x[:, :2]
    for bad in (x[:, 0], x[None]):
        for call in (lambda: ss.ss_attention_packed(bad, k, k, nodes, 3), lambda: ss.ss_attention_packed(x, bad, k, nodes, 3),
                     lambda: ss.ss_attention_packed(x, k, bad, nodes, 3), lambda: ss.ss_attention_packed(x, k, k, nodes, 3, out=bad),
                     lambda: ss.ss_attention_tree(bad, H.cache, context, 40, nodes=nodes, max_nodes=3), lambda: ss.ss_cache_write(H.cache, bad, k, seq, slot),
                     lambda: ss.ss_cache_write(H.cache, k, bad, seq, slot), lambda: ss.ss_cache_read(H.cache, seq, slot, k=bad)):
            with pytest.raises(ValueError, match="must be"):
                call()


@pytest.mark.parametrize("nodes,group,dim,context", [(1, 1, 128, 3900), (1, 16, 64, 700), (4, 4, 128, 300), (16, 1, 64, 60)])
@pytest.mark.parametrize("lowest", [0, 3, 20])
def test_half_results_of_few_rows_over_8_bits_have_one_rounding(nodes, group, dim, context, lowest):
    """Up to 16 rows a unit weights are pairs of halves: off by 2^-22 of themselves (2^-11 of what the first leaves, 2^-11), or where they are
    subnormal by 2^-25 R with 2^6 R at most the largest product, times codes up to 127.  Scores are whole numbers of powers of two from 0 to
    -20, exact but for scale log2(e), which is 1 within 2^-23: 20 2^-23 ln 2 of a weight, 2^-18 with the exponential and the sums."""
    H = Held(126, [context + nodes], 1, dim, I8)
    H.raw["k"].zero_()
    H.raw["k"][:, 0] = -torch.randint(0, lowest + 1, (len(H.raw["k"]),), device="cuda", generator=gen(127)).to(I8)
    H.raw["k_scale"].fill_(1)
    q = torch.zeros(nodes, group, dim, dtype=F16, device="cuda")
    q[..., 0] = 1
    got = ss.ss_attention_tree(q, H.cache, i32([context]), context, nodes=i32([0, nodes]), max_nodes=nodes, scale=math.log(2))
    at = slice(int(H.start[0]), int(H.start[0]) + context + nodes)
    v, unit = H.rows("v", 0, 0, context + nodes), H.raw["v_scale"].double()[at]
    p = torch.exp2(H.raw["k"][at, 0].double()).expand(nodes, -1) * torch.ones(nodes, context + nodes, device="cuda").tril(context)
    w = p / p.sum(-1, keepdim=True)
    ref, A = w @ v, w @ v.abs()
    tol = half_step(F16) * ref.abs() + (2.0 ** -22 + 2.0 ** -18) * A + len(v) * 2.0 ** -31 * 127 * (w * unit).amax(-1, keepdim=True)
    bad = (got.double() - ref[:, None]).abs() > tol[:, None]
    assert not bad.any(), (bad.sum().item(), ((got.double() - ref[:, None]).abs() / tol[:, None]).max().item())

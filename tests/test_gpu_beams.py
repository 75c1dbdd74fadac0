"""Beam search against its definition in 64 bits, and a search over a cache in pages against one that keeps every history apart.

How near a sum is.  log sum exp: an exponential is off by 2^-23 of itself and, by its argument's rounding, by |x| 2^-24 e^x <= 2^-25 of the largest;
a thread adds 32 of them in float32, lanes and waves 8 more: 40 * 2^-24, all in all below 2^-18 (relative of the sum, absolute of its logarithm).  The sum
itself is rounded to float32, 2^-24 of it, its parts are exact.  Candidates whose ranks are nearer to each other than twice that may change
places; exact ties (the same logits, the same beams) may not."""
import math

import numpy as np
import pytest
import torch

from paper_2305_13144_amd import binding as ss
from test_gpu_operators import BF16, F16, gen, i32, randn

pytestmark = pytest.mark.gpu

F32 = torch.float32


def u8(v):
    return torch.tensor(v, dtype=torch.uint8, device="cuda")


def candidates(x, totals, lengths, ended, end_id, power):
    """Of one group: ranks and sums [beams * vocab] in 64 bits, -inf where there is no candidate."""
    beams, vocab = x.shape
    rank, total = np.full((beams, vocab), -np.inf), np.full((beams, vocab), -np.inf)
    for b in range(beams):
        if not np.isfinite(totals[b]):
            continue
        n = 0 if lengths is None else max(lengths[b], 0)
        if ended is not None and ended[b]:
            total[b, max(end_id, 0)] = totals[b]
            rank[b, max(end_id, 0)] = totals[b] / max(n, 1) ** power
            continue
        ok = np.isfinite(x[b])
        if not ok.any():
            continue
        top = x[b][ok].max()
        total[b, ok] = totals[b] + ((x[b][ok] - top) - math.log(np.exp(x[b][ok] - top).sum()))
        rank[b, ok] = total[b, ok] / (n + 1) ** power
    return rank.reshape(-1), total.reshape(-1)


def check(logits, totals, keep, lengths=None, ended=None, end_id=-1, power=0.0, history=None, exact=False, out=None):
    groups, beams = totals.shape
    vocab = logits.shape[1]
    got = ss.ss_beam_select(logits, totals, keep, lengths, ended, end_id, power, history, out)
    x, old = logits.double().cpu().numpy(), totals.double().cpu().numpy()
    ln = None if lengths is None else lengths.view(groups, beams).tolist()
    en = None if ended is None else ended.view(groups, beams).tolist()
    parent, token = got.parent.view(groups, keep).tolist(), got.token.view(groups, keep).tolist()
    sums = got.totals.double().cpu().numpy()
    for g in range(groups):
        l, e = ln and ln[g], en and en[g]
        rank, total = candidates(x[g * beams:(g + 1) * beams], old[g], l, e, end_id, power)
        order = np.argsort(-rank, kind="stable")[:keep]
        order = [int(i) for i in order if rank[i] > -np.inf]
        seen = set()
        for k in range(keep):
            at = g * keep + k
            if k >= len(order):
                assert (parent[g][k], token[g][k], sums[g][k], bool(got.ended[at])) == (-1, -1, -np.inf, True)
                assert got.lengths is None or got.lengths[at] == 0
                assert got.history is None or (got.history[at] == -1).all()
                continue
            b = parent[g][k] - g * beams
            assert 0 <= b < beams
            over = bool(e and e[b])
            assert token[g][k] == end_id if over else 0 <= token[g][k] < vocab
            i = b * vocab + max(token[g][k], 0)
            assert i not in seen
            seen.add(i)
            near = 2.0 ** -18 + 2.0 ** -23 * abs(total[order[k]])
            if exact:
                assert i == order[k], (g, k)
            scale = max((0 if l is None else max(l[b], 0)) + (not over), 1) ** power
            assert abs(rank[i] - rank[order[k]]) <= 2 * near / min(scale, 1.0) + 1e-300, (g, k, rank[i], rank[order[k]])
            assert abs(sums[g][k] - total[i]) <= (2.0 ** -24 * abs(total[i]) if over else near)
            assert bool(got.ended[at]) == (over or token[g][k] == end_id)
            if got.lengths is not None:
                assert got.lengths[at] == max(l[b], 0) + (not over)
            if history is not None:
                width, n = got.history.shape[1], max(l[b], 0)
                want = [-1] * width
                kept = history[g * beams + b].tolist()[:n]
                want[:min(len(kept), width)] = kept[:width]
                if not over and n < width:
                    want[n] = token[g][k]
                assert got.history[at].tolist() == want
    return got


def state(seed, groups, beams, width=0):
    r = np.random.default_rng(seed)
    totals = -torch.rand(groups, beams, device="cuda", generator=gen(seed)) * 30
    lengths = i32(r.integers(0, max(width, 20), groups * beams).tolist())
    ended = u8((r.random(groups * beams) < 0.25).astype(int).tolist())
    history = None
    if width:
        history = i32(r.integers(0, 1000, (groups * beams, width)).tolist())
    return totals, lengths, ended, history


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [1, 2, 7, 255, 1024, 8191, 8192, 8193, 32000, 100003])
def test_vocabularies_of_every_size(dtype, vocab):
    x = (randn(gen(vocab), 6, vocab) * 3).to(dtype)
    totals, lengths, ended, history = state(vocab, 2, 3, 40)
    check(x, totals, 3, lengths, ended, vocab // 2, 0.7, history)


@pytest.mark.parametrize("groups,beams,keep", [(1, 1, 1), (1, 1, 5), (3, 4, 4), (2, 8, 3), (5, 2, 16), (1, 64, 64), (2, 33, 20), (40, 5, 5)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_groups_and_beams(groups, beams, keep, dtype):
    x = (randn(gen(beams), groups * beams, 9001) * 2).to(dtype)
    totals, lengths, ended, history = state(groups, groups, beams, 17)
    check(x, totals, keep, lengths, ended, 5, 1.0, history)
    check(x, totals, keep)
    check(x, totals, keep, ended=ended, end_id=9000)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("shift", [1, 2, 3, 5, 7])
def test_rows_that_begin_anywhere(dtype, shift):
    vocab = 8200 + shift
    wide = torch.full((8 * (vocab + shift) + 16,), 1e4, device="cuda", dtype=dtype)   # what is beside the rows would win
    x = wide[shift:shift + 8 * (vocab + shift)].view(8, vocab + shift)[:, :vocab]
    x.copy_(randn(gen(shift), 8, vocab) * 3)
    check(x, state(shift, 2, 4)[0], 4)


def test_equal_candidates_in_order_of_their_numbers():
    x = torch.zeros(2, 20000, device="cuda")
    totals = torch.zeros(1, 2, device="cuda")
    got = check(x, totals, 64, exact=True)
    assert got.token.tolist() == list(range(64)) and set(got.parent.tolist()) == {0}
    x[:, ::2] = -math.inf
    assert check(x, totals, 64, exact=True).token.tolist() == list(range(1, 128, 2))
    x = torch.zeros(3, 20000, device="cuda", dtype=F16)
    x[:, 19990:] = 2
    x[:, 17] = 2
    got = check(x, torch.tensor([[-1.0, -1.0, -1.0]], device="cuda"), 30, exact=True)
    assert got.token.tolist() == ([17] + list(range(19990, 20000))) * 2 + [17] + list(range(19990, 19997))
    assert got.parent.tolist() == [0] * 11 + [1] * 11 + [2] * 8
    # few distinct values: many ties inside and across chunks and beams with the same sums
    x = torch.randint(0, 4, (1, 30000), device="cuda", generator=gen(1)).float().repeat(4, 1)
    for keep in (1, 7, 64):
        check(x, torch.full((1, 4), -3.0, device="cuda"), keep, exact=True)
        check(x.to(BF16), torch.full((1, 4), -3.0, device="cuda"), keep, exact=True)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("keep", [1, 4, 64])
def test_zeros_of_either_sign_are_equal(dtype, keep):
    """More of them in a wave than its list holds, and than are taken."""
    x = torch.zeros(16, 20000, device="cuda", dtype=dtype)
    x[:, ::2] = -0.0
    assert check(x[:1], torch.zeros(1, 1, device="cuda"), keep, exact=True).token.tolist() == list(range(keep))
    check(x, torch.zeros(1, 16, device="cuda"), keep, exact=True)
    # half of them multiplied by a mask of 0
    x = -randn(gen(keep), 2, 30000).abs().to(dtype) * (torch.rand(2, 30000, device="cuda", generator=gen(1)) < 0.5)
    check(x, torch.full((1, 2), -3.0, device="cuda"), keep, exact=True)


def test_ended_beams_with_sums_of_either_zero_are_equal():
    x = torch.zeros(4, 100, device="cuda")
    for keep in (1, 2, 3):
        got = check(x, torch.tensor([[-0.0, 0.0, 0.0, -0.0]], device="cuda"), keep, ended=u8([1] * 4), end_id=7, exact=True)
        assert got.parent.tolist() == list(range(keep))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_logits_that_are_not_finite_are_no_candidates(dtype):
    x = (randn(gen(1), 8, 9000) * 2).to(dtype)
    x[0] = -math.inf
    x[1, :8999] = math.nan
    x[2, 5], x[2, 6] = math.inf, math.nan
    x[3] = math.nan
    x[4, 100:] = -math.inf
    x[5, :] = math.inf
    totals = torch.tensor([[-1.0, -2.0, -3.0, -4.0], [-1.0, -2.0, -math.inf, math.nan]], device="cuda")
    check(x, totals, 8)
    check(x[4:], totals[1:], 64)                                          # 100 candidates and one beam more
    check(x[4:], totals[1:], 64, ended=u8([0, 1, 1, 1]), end_id=3)
    alone = torch.full((2, 50), -math.inf, device="cuda", dtype=dtype)
    alone[0, 7] = 1
    got = check(alone, torch.zeros(1, 2, device="cuda"), 3, exact=True)
    assert got.token.tolist() == [7, -1, -1] and got.totals[0, 0] == 0


def test_extreme_logits():
    x = torch.tensor([[3e38, 1.0, -3e38, 0.0], [-3e38, -3e38, -3.1e38, -3e38]], device="cuda")
    got = ss.ss_beam_select(x, torch.zeros(1, 2, device="cuda"), 8)
    assert got.parent.tolist() == [0, 1, 1, 1, 1, 0, 0, 0] and got.token.tolist() == [0, 0, 1, 3, 2, 1, 3, 2]
    assert got.totals[0, 0] == 0 and abs(got.totals[0, 1].item() + math.log(3)) < 1e-6
    x = torch.zeros(1, 5000, device="cuda")
    x[0, 4999] = 200.0                                                    # all the others together weigh nothing
    got = check(x, torch.tensor([[-5.0]], device="cuda"), 2, exact=True)
    assert got.token.tolist() == [4999, 0]


@pytest.mark.parametrize("power", range(22, 32))
def test_logits_so_large_that_few_numbers_lie_between_them(power):
    """The largest logits of rows behind a wave's first steps, one to eight units above the rest."""
    unit = 2.0 ** (power - 23)
    x = torch.full((16, 20000), 2.0 ** power, device="cuda")
    for b in range(16):
        x[b] += unit * (b % 2)
        x[b, 19000 + b] += unit * (1 + b // 2)
    x[8:] = -x[8:].flip(1)
    x[8:, 19999] = -2.0 ** power + unit * 4
    check(x, torch.linspace(-0.5, -8.0, 16, device="cuda")[None], 64)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("kind", ["late", "early", "ascending", "descending"])
def test_how_near_the_sum_of_exponentials_is(dtype, kind):
    """Rows of zeros with a peak behind a wave's first steps or in them, and rows in order.  An exponential is off by 2^-23 of itself, and three additions of those
    of 16 bytes by 2^-24 each: 5 * 2^-24 of the sum.  The argument, x log2 e with x = logit - largest so far, is a rounded difference times a rounded constant
    (2^-26.2 of it), rounded: |x| (2 + 2^-2.2) 2^-24, which counts by the term's share of the sum.  What is in float64 adds nothing that counts; a sum is
    rounded to float32, 2^-24 of it.  No log probability is above 0."""
    if kind in ("late", "early"):
        tops = [0.25, 0.75, 0.875, 1.0, 1.5, 3.0, 5.0, 7.5, 10.0, 14.0, 20.875, 30.0, 40.0, 60.0, 79.0, 79.5]
        x = torch.zeros(16, 32000, device="cuda", dtype=dtype)
        for b, top in enumerate(tops):
            x[b, 31000 - 7 * b if kind == "late" else 7 * b] = top
    else:
        x = (torch.arange(32000, device="cuda") * torch.logspace(-6, -2, 16, device="cuda")[:, None]).to(dtype)
        x = x if kind == "ascending" else x.flip(1).contiguous()
    got = ss.ss_beam_select(x, torch.zeros(1, 16, device="cuda"), 64)
    logp = torch.log_softmax(x.double(), 1)
    off = (logp.exp() * (x.double().amax(1, keepdim=True) - x.double())).sum(1)
    parent = got.parent.long()
    want = logp[parent, got.token.long()]
    assert (parent >= 0).all() and (got.totals <= 0).all()
    assert ((got.totals[0].double() - want).abs() <= 2.0 ** -24 * (5 + 2.25 * off[parent]) + 2.0 ** -24 * want.abs()).all()
    alone = ss.ss_beam_select(x, torch.zeros(16, 1, device="cuda"), 1)                 # each row's largest, its parts in several workgroups
    want = logp.amax(1)
    assert (alone.totals <= 0).all()
    assert ((alone.totals[:, 0].double() - want).abs() <= 2.0 ** -24 * (5 + 2.25 * off) + 2.0 ** -24 * want.abs()).all()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [3, 700, 40000])
def test_logits_that_are_masked_with_the_lowest_number_are_candidates_far_behind(dtype, vocab):
    low = torch.finfo(dtype).min
    x = torch.full((4, vocab), low, device="cuda", dtype=dtype)
    x[1, vocab - 1] = 2.0                                                 # all but one
    x[2, : vocab // 2] = randn(gen(1), vocab // 2).to(dtype)              # half of them
    x[3, ::2] = -math.inf                                                 # the others are no candidates at all
    got = check(x, torch.tensor([[-1.0], [-2.0], [-3.0], [-4.0]], device="cuda"), 2)
    for row, n in ((0, vocab), (3, vocab // 2)):                          # whole rows of the lowest number: all alike
        assert got.totals[row, 0].isfinite() and abs(got.totals[row, 0].item() + (1.0, 2.0, 3.0, 4.0)[row] + math.log(n)) <= 2.0 ** -18 + 2.0 ** -24 * 20
    assert got.token.view(4, 2)[0].tolist() == [0, 1] and got.totals[1, 0] == -2.0 and got.token.view(4, 2)[1].tolist() == [vocab - 1, 0]


def test_ended_beams_stay_with_their_sum():
    x = torch.zeros(4, 100, device="cuda")
    totals = torch.tensor([[-1.0, -0.5, -9.0, -9.0]], device="cuda")
    got = check(x, totals, 4, i32([3, 4, 5, 6]), u8([1, 0, 1, 0]), 42, 1.0, i32(np.arange(40).reshape(4, 10).tolist()))
    assert got.token[0] == 42 and got.parent[0] == 0 and got.lengths[0] == 3 and got.ended[0] == 1
    got = check(x, totals, 3, i32([3, 4, 5, 6]), u8([1, 1, 1, 1]), -1, 1.0)
    assert got.token.tolist() == [-1] * 3 and got.parent.tolist() == [1, 0, 3]
    got = check(x, totals, 6, i32([0, 0, 0, 0]), u8([1, 1, 1, 1]), 9, 2.0)
    assert got.parent.tolist() == [1, 0, 2, 3, -1, -1]


def test_a_power_below_all_numbers_leaves_sums_of_zero_first():
    """10^-400 is 0 in float64, and 0 / 0 no rank."""
    x = torch.full((3, 5), -math.inf, device="cuda")
    x[0, 1] = x[1, 2] = x[2, 3] = 1.0
    totals = torch.tensor([[0.0, -1.0, 0.0]], device="cuda")
    got = ss.ss_beam_select(x, totals, 4, i32([9, 9, 9]), length_power=-400.0)
    assert got.parent.tolist() == [0, 2, 1, -1] and got.token.tolist() == [1, 3, 2, -1]
    assert got.totals.tolist() == [[0.0, 0.0, -1.0, -math.inf]]


def test_histories_without_room_and_of_another_width():
    x = randn(gen(1), 4, 50)
    totals, lengths, ended, history = state(3, 1, 4, 6)
    lengths = i32([6, 5, -3, 2**31 - 1])
    ended = u8([0, 0, 0, 1])
    n = 4
    for width in (0, 1, 4, 6, 9):
        out = ss.Beams(i32([9] * n), i32([9] * n), torch.zeros(1, n, device="cuda"), i32([9] * n), u8([9] * n), torch.full((n, width), 9, dtype=torch.int32, device="cuda"))
        if width:
            check(x, totals, n, lengths, ended, 3, 0.0, history, out=out)


def test_the_largest_number_of_rows():
    x = randn(gen(1), 65535, 37)
    totals = -torch.rand(65535, 1, device="cuda", generator=gen(2))
    got = ss.ss_beam_select(x, totals, 2)
    best = torch.sort(x, dim=1, descending=True, stable=True)
    assert torch.equal(got.token.view(-1, 2), best.indices[:, :2].int()) and torch.equal(got.parent.view(-1, 2), i32(list(range(65535)))[:, None].expand(-1, 2))
    want = totals.double() + torch.log_softmax(x.double(), 1).gather(1, best.indices[:, :2])
    assert ((got.totals.double() - want).abs() <= 2.0 ** -18 + 2.0 ** -23 * want.abs()).all()
    got = ss.ss_beam_select(x[:65472], totals.view(-1)[:65472].view(1023, 64), 64)
    want = (totals.view(-1)[:65472, None].double() + torch.log_softmax(x[:65472].double(), 1)).view(1023, -1).sort(1, descending=True).values[:, :64]
    assert ((got.totals.double() - want).abs() <= 2.0 ** -18 + 2.0 ** -23 * want.abs()).all()


def test_new_rows_of_a_search_begin_from_one_beam():
    x = randn(gen(2), 3, 4000)
    got = check(x, torch.zeros(3, 1, device="cuda"), 5)
    for g in range(3):
        assert got.token.view(3, 5)[g].tolist() == torch.sort(x[g], descending=True).indices[:5].tolist()


def test_the_same_call_gives_the_same_bits_in_graphs():
    x = (randn(gen(5), 64, 50001) * 2).to(BF16)
    totals, lengths, ended, history = state(5, 8, 8, 30)
    def call():
        return ss.ss_beam_select(x, totals, 8, lengths, ended, 7, 0.6, history)
    first = [t.clone() for t in call()]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = call()
    for _ in range(3):
        for t in held:
            t.fill_(3)
        g.replay()
        torch.cuda.synchronize()
        again = call()
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(first, held, again))
    s = torch.cuda.Stream()
    got = ss.ss_beam_select(x, totals, 8, lengths, ended, 7, 0.6, history, stream=s.cuda_stream)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, got))


# ------------------------------------------------------------------------------------------------ a search over pages
class Toy:
    """A model of two attention layers, without any order of its own beyond what the cache holds: enough that a wrong page shows."""

    def __init__(self, seed, kv, each, dim, vocab, dtype):
        g = gen(seed)
        self.kv, self.heads, self.dim, self.vocab, self.dtype = kv, kv * each, dim, vocab, dtype
        d = self.heads * dim
        self.embed = randn(g, vocab, d) / 2
        self.wk, self.wv, self.wq = ([randn(g, d, n * dim) * d ** -0.5 * f for _ in range(2)] for n, f in ((kv, 2.0), (kv, 1.0), (self.heads, 2.0)))
        self.head = randn(g, d, vocab) * d ** -0.5 * 4

    def qkv(self, layer, x):
        return [(x @ w[layer]).view(len(x), -1, self.dim).to(self.dtype) for w in (self.wq, self.wk, self.wv)]

    def logits(self, x):
        return x @ self.head

    def whole(self, tokens):
        """Logits behind the last of a row's tokens, everything computed anew: what a search without a cache does."""
        x = self.embed[tokens]
        for layer in range(2):
            q, k, v = self.qkv(layer, x)
            k, v, q = (t.double().repeat_interleave(self.heads // t.shape[1], 1).transpose(0, 1).contiguous() for t in (k, v, q))
            s = q @ k.transpose(1, 2).contiguous() * self.dim ** -0.5
            s = s.masked_fill(torch.ones(s.shape[1:], dtype=torch.bool, device="cuda").triu(1), -math.inf)
            x = x + (torch.softmax(s, -1) @ v).transpose(0, 1).reshape(len(tokens), -1).float()
        return self.logits(x[-1:])


@pytest.mark.parametrize("page,beams,kv,each,dtype", [(16, 4, 2, 2, F16), (32, 3, 1, 4, F16), (16, 8, 2, 1, BF16)])
def test_a_search_over_pages(page, beams, kv, each, dtype):
    """Select, fork, copy, write and attend, step after step, with a compaction on the way; every step's logits against those of the whole histories."""
    dim, vocab, width, steps, end = 64, 60, 80, 24, 0
    m = Toy(page, kv, each, dim, vocab, dtype)
    r = np.random.default_rng(page)
    prompts = [[int(x) for x in r.integers(1, vocab, n)] for n in (page + 3, 5, page, 2)]
    groups, n_pages = len(prompts), 4 * len(prompts) * beams + 20
    rows, stride = groups * beams, -(-width // page) + 1
    layers = [ss.Pages.allocate(n_pages, page, kv, dim, dtype) for _ in range(2)]
    tables = [ss.PageTable.allocate(rows, stride, page, n_pages) for _ in range(2)]
    one = ss.PageTable.allocate(groups, stride, page, n_pages)
    now = ss.PageTable.allocate(groups, stride, page, n_pages)
    # the prompts: each its pages, all tokens at once
    _, _, missing = ss.ss_pages_fork(one, now, grow=i32([len(p) for p in prompts]), parent=i32([-1] * groups))
    flat, offsets = sum(prompts, []), np.cumsum([0] + [len(p) for p in prompts])
    row = i32(np.repeat(np.arange(groups), [len(p) for p in prompts]).tolist())
    pos = i32(sum([list(range(len(p))) for p in prompts], []))
    x = m.embed[flat]
    for layer in range(2):
        q, k, v = m.qkv(layer, x)
        ss.ss_pages_write(layers[layer], now, k, v, row, pos)
        out = ss.ss_attention_packed(q, k, v, i32(offsets.tolist()), max(len(p) for p in prompts))
        x = x + out.float().view(len(flat), -1)
    logits = m.logits(x[(offsets[1:] - 1).tolist()])
    history = torch.full((groups, width), -1, dtype=torch.int32, device="cuda")
    for g, p in enumerate(prompts):
        history[g, :len(p)] = i32(p)
    state = ss.Beams(None, None, torch.zeros(groups, 1, device="cuda"), i32([len(p) for p in prompts]), u8([0] * groups), history)
    worst = 0.0
    for step in range(steps):
        state = ss.ss_beam_select(logits, state.totals, beams, state.lengths, state.ended, end, 0.7, state.history)
        src, dst, missing = ss.ss_pages_fork(now, tables[step % 2], state.parent, (1 - state.ended.int()).contiguous())
        ss.ss_pages_copy(layers, src, dst)
        now = tables[step % 2]
        assert missing.item() == 0
        if step == 11:
            src, dst, _, counts = ss.ss_pages_compact(now)
            ss.ss_pages_copy(layers, src, dst, counts[1:])
        x = m.embed[state.token.long().clamp_min(0)]
        live = torch.nonzero(state.ended == 0).view(-1).tolist()
        at = torch.where(state.ended == 0, now.lengths - 1, -1)
        for layer in range(2):
            q, k, v = m.qkv(layer, x)
            ss.ss_pages_write(layers[layer], now, k, v, i32(list(range(rows))), at)
            x = x + ss.ss_attention_pages(q, layers[layer], now, width, beams).float().view(rows, -1)
        logits = m.logits(x)
        for i in live[step % 3::3]:
            tokens = state.history[i, :state.lengths[i]].tolist()
            assert min(tokens) >= 0
            want = m.whole(tokens)[0]
            worst = max(worst, ((logits[i] - want).abs().max() / want.abs().max()).item())
    # two layers, each with a result rounded to 16 bits (half a step) and weights likewise, the logits about as large as what comes in: four roundings
    # a layer, each seen through the next layer's keys and values once more
    assert worst <= 16 * torch.finfo(dtype).eps

"""Caches in pages against their definitions: tokens into and out of pages, attention over them in 64 bits (tolerances as derived in
test_gpu_operators.py), tables that fork, grow, end and are made dense against a plain implementation that handles one page at a time, and the copies
that follow from those."""
import math

import numpy as np
import pytest
import torch

from paper_2305_13144_amd import binding as ss
from test_gpu_operators import BF16, F16, I8, assert_attention, codes_of, gen, half_step, i32, randn

pytestmark = pytest.mark.gpu


def pool_of(seed, n_pages, page, kv, dim, held):
    """Pages full of random vectors, and what they stand for in 64 bits [pages, kv, page, dim]."""
    g, parts, values = gen(seed), [], []
    for _ in range(2):
        x = randn(g, n_pages, kv, page, dim)
        if held == I8:
            x = x * torch.exp(0.5 * randn(g, n_pages, kv, page, 1))
            unit = x.abs().amax(-1) / 127
            parts.append((torch.round(x / unit[..., None]).to(I8), unit))
            values.append(parts[-1][0].double() * unit[..., None].double())
        else:
            parts.append((x.to(held), None))
            values.append(parts[-1][0].double())
    (k, ks), (v, vs) = parts
    flat = [None if t is None else t.reshape(-1) for t in (k, v, ks, vs)]
    return ss.Pages(flat[0], flat[1], page, kv, dim, flat[2], flat[3]), values


def table_of(rows, lengths, stride, page, n_pages, fill=-1):
    t = np.full((len(rows), stride), fill, np.int32)
    for i, r in enumerate(rows):
        t[i, :len(r)] = r
    return ss.PageTable(i32(t.tolist()).view(len(rows), stride), i32(lengths), page, n_pages)


# ------------------------------------------------------------------------------------------------ write and read
@pytest.mark.parametrize("n", [1, 3, 70])
@pytest.mark.parametrize("kv,dim", [(1, 64), (4, 64), (8, 128), (5, 128)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("held,page", [(I8, 16), (F16, 32), (BF16, 256)])
def test_tokens_go_to_the_pages_of_their_positions_and_come_back(n, kv, dim, dtype, held, page):
    g, r = gen(n), np.random.default_rng(n)
    lengths = [page + 5, 0, 2 * page, 3]
    pages = ss.Pages.allocate(9, page, kv, dim, held)
    for x in (pages.k, pages.v):
        x.fill_(3)
    table = table_of([[7, 2, 5], [1], [0, 8], [-1]], lengths, 3, page, 9)     # row 3 has no page, row 0 one behind its length
    wide = randn(g, n, 3 * kv + 2, dim, dtype=dtype)                          # keys and values are views of a wider projection
    k, v = wide[:, 1:1 + kv], wide[:, 2 + kv:2 + 2 * kv]
    places = [(0, s) for s in range(page + 5)] + [(2, s) for s in range(2 * page)]
    pick = r.permutation(len(places))[:n]
    n = len(pick)
    row, pos = [places[i][0] for i in pick], [places[i][1] for i in pick]
    if n > 2:
        row[0], pos[1] = -1, 2 * page
        if n > 25:
            for at, x in zip(range(10, 17), [(4, 0), (0, -1), (0, page + 5), (1, 0), (3, 1), (2, 2**31 - 1), (-2**31, 0)]):
                row[at], pos[at] = x
    here = [t for t in range(n) if (row[t], pos[t]) in places]
    ss.ss_pages_write(pages, table, k[:n], v[:n], i32(row), i32(pos))
    rk, rv = (torch.full((n, kv, dim), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    ss.ss_pages_read(pages, table, i32(row), i32(pos), k=rk, v=rv)
    number = {(0, 0): 7, (0, 1): 2, (2, 0): 0, (2, 1): 8}
    for x, back, store, unit in ((k[:n], rk, pages.k, pages.k_scale), (v[:n], rv, pages.v, pages.v_scale)):
        want = torch.full_like(store, 3).view(-1, dim)
        at = torch.tensor([[(number[row[t], pos[t] // page] * kv + h) * page + pos[t] % page for h in range(kv)] for t in here], dtype=torch.int64,
                          device="cuda").view(len(here), kv)
        if held == I8:
            scale, codes = codes_of(x)
            want[at] = torch.tensor(codes, device="cuda")[here]
            assert torch.equal(unit[at].cpu(), torch.tensor(scale)[here])
            value = (torch.tensor(codes).float() * torch.tensor(scale)[..., None]).to(dtype)
        else:
            want[at] = x[here].to(held)
            value = x.to(held).to(dtype).cpu()
        assert torch.equal(store.view(-1, dim), want)                         # the rest of the pool is as it was
        wanted = torch.full((n, kv, dim), 7.0, dtype=dtype)
        wanted[here] = value[here]
        assert torch.equal(back.cpu(), wanted)                                # and so are rows of tokens that do not exist


@pytest.mark.parametrize("page", [16, 64])
def test_without_a_list_each_row_gets_its_last_position(page):
    pages = ss.Pages.allocate(6, page, 2, 64, F16)
    table = table_of([[3, 1], [4], [], [5], [0, 2]], [page + 1, page, 0, 1, 2 * page + 9], 2, page, 6)   # the last is longer than its entries
    k, v = randn(gen(1), 5, 2, 64, dtype=F16), randn(gen(2), 5, 2, 64, dtype=F16)
    ss.ss_pages_write(pages, table, k, v)
    rk, rv = ss.ss_pages_read(pages, table, k=torch.zeros_like(k), v=torch.zeros_like(v))
    live = [0, 1, 3, 4]
    assert torch.equal(rk[live], k[live]) and torch.equal(rv[live], v[live]) and not rk[2].any()
    held = pages.k.view(6, 2, page, 64)
    for row, (p, s) in {0: (1, 0), 1: (4, page - 1), 3: (5, 0), 4: (2, page - 1)}.items():
        assert torch.equal(held[p, :, s], k[row])
    assert int((held != 0).any(-1).any(1).sum()) == 4
    ss.ss_pages_write(pages, table, k[:2] * 2, v[:2])                        # of the first rows only
    assert torch.equal(held[1, :, 0], k[0] * 2) and torch.equal(held[5, :, 0], k[3])


# ------------------------------------------------------------------------------------------------ attention
def random_rows(r, lengths, page, group=1, agree=0.6, room=3):
    """Pages of rows, where rows of a group hold the same ones at first; how many pages there are, and entries."""
    taken, rows = 0, []
    for i, n in enumerate(lengths):
        need = -(-n // page)
        mine = rows[-1][:int(need * agree)] if i % group else []
        mine = list(mine)
        while len(mine) < need:
            mine.append(taken)
            taken += 1
        rows.append(mine)
    n_pages = taken + 3
    place = r.permutation(n_pages)
    return [[int(place[x]) for x in m] for m in rows], n_pages, max([1] + [len(m) for m in rows]) + room


def check_attention(seed, lengths, page, kv, heads_each, dim, dtype, held, group=1, agree=0.6, scale=None, max_length=None, holes=0, pick=None, spoil=True, out=None):
    r = np.random.default_rng(seed)
    rows, n_pages, stride = random_rows(r, lengths, page, group, agree)
    pages, (k, v) = pool_of(seed, n_pages, page, kv, dim, held)
    for _ in range(holes):                                    # entries that are no page
        i = int(r.integers(len(rows)))
        if rows[i]:
            rows[i][int(r.integers(len(rows[i])))] = int(r.choice([-1, n_pages, 2**31 - 1, -2**31]))
    n_rows = len(rows)
    seen = torch.zeros(n_pages, page, dtype=torch.bool)
    for m, n in zip(rows, lengths):
        for e, p in enumerate(m):
            if 0 <= p < n_pages:
                seen[p, :max(min(page, n - e * page), 0)] = True
    if spoil:                                                 # what no row sees is as bad as can be
        bad = (~seen).cuda()[:, None, :].expand(n_pages, kv, page)
        for x, unit in ((pages.k, pages.k_scale), (pages.v, pages.v_scale)):
            if held == I8:
                unit.view(n_pages, kv, page)[bad] = math.nan
            else:
                x.view(n_pages, kv, page, dim)[bad] = math.nan
    table = table_of(rows, lengths, stride, page, n_pages, fill=n_pages - 1)   # entries behind a length are not looked at
    heads, n = kv * heads_each, n_rows if pick is None else len(pick)
    q = randn(gen(seed + 1), n, heads + 2, dim, dtype=dtype)[:, 1:1 + heads]
    if out == "wide":
        out = torch.full((n + 1, heads, dim + 8), 5.0, dtype=dtype, device="cuda")
        got = ss.ss_attention_pages(q, pages, table, max(lengths + [0]) if max_length is None else max_length, group, None if pick is None else i32(pick), scale, out[:n, :, :dim])
        assert (out[n:] == 5).all() and (out[:, :, dim:] == 5).all()
    else:
        got = ss.ss_attention_pages(q, pages, table, max(lengths + [0]) if max_length is None else max_length, group, None if pick is None else i32(pick), scale)
    scale = dim ** -0.5 if scale is None else scale
    for j in range(n):
        i = j if pick is None else pick[j]
        if not 0 <= i < n_rows or lengths[i] < 1:
            assert not got[j].any()
            continue
        m = torch.tensor(rows[i], device="cuda")
        real = (m >= 0) & (m < n_pages)
        m = torch.where(real, m, 0)
        visible = (real[:, None] & torch.ones(page, dtype=torch.bool, device="cuda")).reshape(-1)[:lengths[i]]
        kk, vv = (x[m].permute(1, 0, 2, 3).reshape(kv, -1, dim)[:, :lengths[i]] for x in (k, v))
        for h in range(kv):
            kh, vh = (torch.where(visible[:, None], x[h], 0.0) for x in (kk, vv))
            assert_attention(got[j, h * heads_each:(h + 1) * heads_each], q[j, h * heads_each:(h + 1) * heads_each], kh, vh,
                             visible.expand(heads_each, -1), scale, F16 if held == I8 else held)
    return got


TYPES = [(F16, F16), (BF16, BF16), (F16, I8), (BF16, I8)]


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype,held", TYPES)
def test_single_rows_of_every_length(page, dim, dtype, held):
    check_attention(page + dim, [1, 0, 15, 16, 17, 31, 32, 33, page - 1, page, page + 1, 2 * page, 700, 129], page, 2, 3, dim, dtype, held)


@pytest.mark.parametrize("kv,each", [(4, 1), (1, 8), (2, 4), (3, 7), (1, 17), (2, 16), (1, 40), (33, 1)])
@pytest.mark.parametrize("dtype,held", TYPES)
def test_heads_that_share_keys_and_values(kv, each, dtype, held):
    check_attention(kv * each, [5, 300, 77], 32, kv, each, 128, dtype, held)


@pytest.mark.parametrize("group,each", [(2, 1), (3, 4), (4, 4), (8, 1), (8, 4), (5, 8), (32, 1), (32, 3), (16, 8)])
@pytest.mark.parametrize("agree", [0.0, 0.7, 1.0])
@pytest.mark.parametrize("dtype,held", [(F16, F16), (BF16, I8)])
def test_rows_that_are_looked_at_together(group, each, agree, dtype, held):
    r = np.random.default_rng(group)
    lengths = [int(n) for n in r.integers(150, 400, 2 * group)]
    lengths[1] = 0
    check_attention(7 * group + each, lengths, 16, 2, each, 64, dtype, held, group, agree)


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("dtype,held", TYPES)
def test_beams_of_long_prompts(page, dtype, held):
    check_attention(page, [3000, 3007, 2990, 3001, 1200, 1250, 1201, 1199], page, 2, 4, 128, dtype, held, 4, 0.9)


@pytest.mark.parametrize("dtype,held", TYPES)
def test_one_long_row_and_many_short_ones(dtype, held):
    check_attention(3, [20011], 64, 4, 2, 128, dtype, held)
    check_attention(4, [9000] + [3] * 40 + [200, 0, 1], 16, 2, 1, 64, dtype, held)
    check_attention(5, [17] * 300, 16, 1, 1, 64, dtype, held)


@pytest.mark.parametrize("rows,group,each,dim,length", [(1, 1, 16, 128, 3900), (4, 4, 8, 128, 300), (32, 32, 1, 64, 700), (8, 8, 4, 64, 60), (2, 1, 40, 128, 129)])
@pytest.mark.parametrize("lowest", [0, 3, 20])
def test_half_results_over_8_bits_have_one_rounding(rows, group, each, dim, length, lowest):
    """However many rows a unit has: weights are pairs of halves, off by 2^-22 of themselves (2^-11 of what the first leaves, 2^-11), or where they are
    subnormal by 2^-25 R with 2^6 R at most the largest product, times codes up to 127.  Scores are whole numbers of powers of two from 0 to
    -20, exact but for scale log2(e), which is 1 within 2^-23: 20 2^-23 ln 2 of a weight, 2^-18 with the exponential and the sums."""
    r = np.random.default_rng(rows)
    lists, n_pages, stride = random_rows(r, [length] * rows, 16, group, 0.8)
    pages, (_, v) = pool_of(126, n_pages, 16, 1, dim, I8)
    pages.k.zero_()
    keys = pages.k.view(n_pages, 16, dim)
    keys[:, :, 0] = -torch.randint(0, lowest + 1, (n_pages, 16), device="cuda", generator=gen(127)).to(I8)
    pages.k_scale.fill_(1)
    q = torch.zeros(rows, each, dim, dtype=F16, device="cuda")
    q[..., 0] = 1
    got = ss.ss_attention_pages(q, pages, table_of(lists, [length] * rows, stride, 16, n_pages), length, group, scale=math.log(2))
    for i, m in enumerate(lists):
        p = torch.exp2(keys[m, :, 0].double()).reshape(-1)[:length]
        vv, unit = v[m, 0].reshape(-1, dim)[:length], pages.v_scale.view(n_pages, 16)[m].double().reshape(-1)[:length]
        w = p / p.sum()
        ref, A = w @ vv, w @ vv.abs()
        tol = half_step(F16) * ref.abs() + (2.0 ** -22 + 2.0 ** -18) * A + length * 2.0 ** -31 * 127 * (w * unit).max()
        assert ((got[i].double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("group", [1, 4])
@pytest.mark.parametrize("dtype,held", TYPES)
def test_entries_that_are_no_page_are_not_seen(group, dtype, held):
    check_attention(9, [300, 280, 270, 290, 50, 16, 17, 40], 16, 2, 2, 64, dtype, held, group, 0.8, holes=30)
    pages, _ = pool_of(1, 3, 16, 2, 64, held)
    q = randn(gen(1), 4, 4, 64, dtype=dtype)
    assert not ss.ss_attention_pages(q, pages, table_of([[-1, -1], [5], [], [-7]], [32, 16, 0, -9], 2, 16, 3), 32, group).any()


@pytest.mark.parametrize("dtype,held", TYPES)
@pytest.mark.parametrize("n,kv,each,dim,top,group", [(150, 16, 1, 64, 9000, 1), (60, 8, 4, 128, 16000, 1), (40, 12, 20, 64, 12000, 1), (64, 16, 2, 64, 9000, 4)])
def test_many_long_rows_of_unlike_length(dtype, held, n, kv, each, dim, top, group):
    """So much that units are cut into large parts and small ones.  Rows take their pages from a small pool, which rows of a table may share."""
    r = np.random.default_rng(n)
    page, n_pages = 64, 300
    pages, (k, v) = pool_of(n, n_pages, page, kv, dim, held)
    lengths = [int(top * x ** 2) for x in r.random(n)]
    lengths[3], lengths[7], lengths[n - 1] = top, 0, 1
    stride = -(-top // page)
    table = r.integers(0, n_pages, (n, stride)).astype(np.int32)
    if group > 1:
        for i in range(n):
            if i % group:
                table[i, :stride // 2] = table[i - 1, :stride // 2]
    q = randn(gen(1), n, kv * each, dim, dtype=dtype)
    tb = ss.PageTable(torch.tensor(table, device="cuda"), i32(lengths), page, n_pages)
    got = ss.ss_attention_pages(q, pages, tb, top, group)
    assert torch.equal(got, ss.ss_attention_pages(q, pages, tb, top, group)) and not got[7].any()
    for i in [i for i in (1, 3, n // 2, n - 1) if lengths[i]]:
        m = torch.tensor(table[i], device="cuda").long()
        kk, vv = (x[m].permute(1, 0, 2, 3).reshape(kv, -1, dim)[:, :lengths[i]] for x in (k, v))
        for h in (0, kv - 1):
            assert_attention(got[i, h * each:(h + 1) * each], q[i, h * each:(h + 1) * each], kk[h], vv[h],
                             torch.ones(each, lengths[i], dtype=torch.bool, device="cuda"), dim ** -0.5, F16 if held == I8 else held)
    few = ss.ss_attention_pages(q, pages, tb, 1, group)          # a workgroup a unit: other sums, the same results but for roundings
    assert ((few.double() - got.double()).abs() <= 4 * half_step(dtype) * (got.double().abs() + v.abs().max() * 0.1)).all()


@pytest.mark.parametrize("group", [1, 5])
@pytest.mark.parametrize("most", [16, 5000])
def test_the_largest_number_of_queries(group, most):
    """65535 rows of one page each; with a longest length that is far too large units are cut by the rows' lengths all the same."""
    n, n_pages = 65535, 50
    pages, (k, v) = pool_of(1, n_pages, 16, 1, 64, F16)
    at = torch.randint(0, n_pages, (n, 1), device="cuda", generator=gen(2)).int()
    lengths = torch.randint(0, 17, (n,), device="cuda", generator=gen(3)).int()
    q = randn(gen(4), n, 1, 64, dtype=F16)
    got = ss.ss_attention_pages(q, pages, ss.PageTable(at, lengths, 16, n_pages), most, group)
    kk, vv = k[at[:, 0].long(), 0], v[at[:, 0].long(), 0]                      # [n, 16, 64]
    score = (kk * q[:, 0, None, :].double()).sum(-1) * 0.125
    score = score.masked_fill(torch.arange(16, device="cuda") >= lengths[:, None], -math.inf)
    w = torch.softmax(score, -1).nan_to_num(0.0)
    want, A = (w[..., None] * vv).sum(1), (w[..., None] * vv.abs()).sum(1)
    tol = half_step(F16) * want.abs() + (half_step(F16) + 2.0 ** -13) * A + 16 * 2.0 ** -23 * v.abs().max()   # as assert_attention; the scores' part is below 2^-14
    assert ((got[:, 0].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("group,n", [(1, 4096), (5, 4095)])
@pytest.mark.parametrize("dtype,held", [(F16, F16), (BF16, I8)])
def test_thousands_of_queries_cut_by_their_rows_lengths(group, n, dtype, held):
    """A lane of a workgroup that looks for its part has many groups here.  The queries share 40 rows, and some have none."""
    r = np.random.default_rng(n)
    page, stride, n_pages, dim = 16, 800, 2000, 64
    pages, (k, v) = pool_of(1, n_pages, page, 1, dim, held)
    lengths = [int(stride * page * x ** 3) for x in r.random(40)]
    lengths[5], lengths[6], lengths[7] = stride * page, 0, 1
    table = r.integers(0, n_pages, (40, stride)).astype(np.int32)
    tb = ss.PageTable(torch.tensor(table, device="cuda"), i32(lengths), page, n_pages)
    pick = r.integers(-1, 41, n)
    pick[::7] = 7
    pick[100:103] = 5
    q = randn(gen(4), n, 1, dim, dtype=dtype)
    most = stride * page
    dealt, whole = (ss.ss_attention_pages_workspace(1, 1, dim, page, stride, n, m, group) for m in (most, 16))
    assert dealt >= whole + n // group * 8 + 1024 * 16 * (dim + 4) * 4      # parts, and notes of where those of each unit lie
    got = ss.ss_attention_pages(q, pages, tb, most, group, rows=i32(pick.tolist()))
    for i in range(-1, 41):
        at = torch.tensor(np.nonzero(pick == i)[0], device="cuda")
        if not 0 <= i < 40 or lengths[i] == 0:
            assert not got[at].any()
            continue
        m = torch.tensor(table[i], device="cuda").long()
        kk, vv = (x[m, 0].reshape(-1, dim)[:lengths[i]] for x in (k, v))
        for a in at.split(512):
            assert_attention(got[a, 0], q[a, 0], kk, vv, torch.ones(len(a), lengths[i], dtype=torch.bool, device="cuda"), dim ** -0.5, F16 if held == I8 else held)


def test_rows_chosen_by_a_list_and_results_with_strides():
    check_attention(11, [100, 37, 250, 1], 32, 2, 2, 128, F16, I8, pick=[2, 0, -1, 2, 4, 3, 2**31 - 1], out="wide")
    check_attention(12, [100, 37, 250, 1], 32, 2, 2, 64, BF16, BF16, group=2, pick=[2, 0, 1, 3, -5, 2], out="wide")


@pytest.mark.parametrize("most", [0, 1, 100, 2**30])
def test_a_wrong_longest_length_only_costs_time(most):
    check_attention(13, [900, 20, 400, 0], 16, 2, 4, 128, F16, F16, max_length=most)
    check_attention(14, [900, 20, 400, 0], 16, 2, 4, 128, BF16, I8, group=2, max_length=most)


@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0, 1e-8])
@pytest.mark.parametrize("dtype,held", TYPES)
def test_scales(scale, dtype, held):
    check_attention(15, [90, 33, 5], 16, 2, 4, 64, dtype, held, scale=scale)


@pytest.mark.parametrize("group", [1, 2])
@pytest.mark.parametrize("held", [F16, BF16, I8])
def test_values_that_are_not_finite_reach_those_who_see_them(group, held):
    dtype = F16 if held == I8 else held
    pages, (_, v) = pool_of(5, 8, 16, 1, 64, held)
    table = table_of([[0, 1, 2], [0, 3, 2]], [48, 40], 3, 16, 8)           # row 1 sees 8 slots of page 2, row 0 all
    q = randn(gen(3), 2, 2, 64, dtype=dtype)
    plain = ss.ss_attention_pages(q, pages, table, 48, group)
    if held == I8:
        pages.v_scale.view(8, 16)[2, 9] = math.nan                         # row 0 only
        got = ss.ss_attention_pages(q, pages, table, 48, group)
        assert got[0].isnan().all()
    else:
        pages.v.view(8, 16, 64)[2, 9, 5] = math.inf
        pages.v.view(8, 16, 64)[3, 1, 7] = math.nan                        # row 1 only
        got = ss.ss_attention_pages(q, pages, table, 48, group)
        assert (got[0, :, 5].abs() >= 65504).all() and got[1, :, 7].isnan().all()        # half saturates
        got[0, :, 5], got[1, :, 7] = plain[0, :, 5], plain[1, :, 7]
        assert got[0].isfinite().all()
    assert got[1].isfinite().all()
    ok = (got[1].double() - plain[1].double()).abs() <= 4 * torch.finfo(dtype).eps * (plain[1].double().abs() + v.abs().max())
    assert ok.all()


@pytest.mark.parametrize("held", [F16, BF16])
@pytest.mark.parametrize("group,each,dim", [(1, 1, 64), (1, 4, 128), (4, 4, 128), (8, 8, 64)])
@pytest.mark.parametrize("most", [1, 700, 2**20])
def test_what_no_row_sees_changes_no_bit(held, group, each, dim, most):
    """Ends of last pages, pages of nobody, and page 0, which stands in for entries that are no page."""
    r = np.random.default_rng(group)
    lengths = [700, 33, 120, 650, 5, 0, 16, 300] * 2
    rows, n_pages, stride = random_rows(r, lengths, 16, group, 0.7)
    rows = [[p + 1 for p in m] for m in rows]
    rows[2][1] = rows[3][7] = rows[3][8] = -1
    n_pages += 1
    stride = max(stride, most // 16)                                       # with room for rows so long
    pages, _ = pool_of(3, n_pages, 16, 2, dim, held)
    unseen = torch.ones(n_pages, 16, dtype=torch.bool)
    for m, n in zip(rows, lengths):
        for e, p in enumerate(m):
            if p > 0:
                unseen[p, :max(min(16, n - e * 16), 0)] = False
    assert unseen[0].all()
    bad = unseen.cuda()[:, None, :].expand(n_pages, 2, 16)
    table = table_of(rows, lengths, stride, 16, n_pages)
    q = randn(gen(1), 16, 2 * each, dim, dtype=held)
    want = ss.ss_attention_pages(q, pages, table, most, group)
    for x in (math.nan, math.inf, 1e4):
        for t in (pages.k, pages.v):
            t.view(n_pages, 2, 16, dim)[bad] = x
        assert torch.equal(ss.ss_attention_pages(q, pages, table, most, group), want)


@pytest.mark.parametrize("held", [F16, BF16])
@pytest.mark.parametrize("each,dim", [(1, 64), (4, 128)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_another_row_sees_changes_no_bit(held, each, dim, bad):
    pages, _ = pool_of(5, 12, 16, 1, dim, held)
    table = table_of([[0, 1, 2, 3], [0, 1, 4, 3], [0, 1, 2, 5], [0, 1, 4, 6]], [60, 49, 50, 51], 4, 16, 12)
    q = randn(gen(3), 4, each, dim, dtype=held)
    want = ss.ss_attention_pages(q, pages, table, 60, 4)
    pages.v.view(12, 16, dim)[3, 5, 9] = bad                               # page 3 is row 0's to slot 11, row 1's to slot 0
    pages.v.view(12, 16, dim)[6, 1, 3] = bad                               # row 3's
    got = ss.ss_attention_pages(q, pages, table, 60, 4)
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    for i, e in ((0, 9), (3, 3)):
        assert (got[i, :, e].isnan() if math.isnan(bad) else got[i, :, e].float() >= 65504).all()      # half saturates
        other = torch.arange(dim, device="cuda") != e
        assert torch.equal(got[i][:, other], want[i][:, other])


@pytest.mark.parametrize("dtype,held", TYPES)
@pytest.mark.parametrize("group,each,dim", [(1, 8, 64), (4, 1, 128), (4, 8, 64), (8, 4, 128)])
@pytest.mark.parametrize("times", [4.0, 300.0, 1e-3])
def test_other_rows_queries_and_keys_change_no_bit(dtype, held, group, each, dim, times):
    """Large scores of one head of a row, and of one row's own pages, move maxima and units of their own only."""
    r = np.random.default_rng(7)
    lengths = [330, 300, 320, 310, 325, 305, 315, 295]
    rows, n_pages, _ = random_rows(r, lengths, 16, group, 0.5)
    pages, _ = pool_of(3, n_pages, 16, 2, dim, held)
    table = table_of(rows, lengths, 2**16, 16, n_pages)
    q = randn(gen(1), 8, 2 * each, dim, dtype=dtype)
    calls = [lambda x, most=most: ss.ss_attention_pages(x, pages, table, most, group) for most in (1, 330, 2**20)]
    want = [f(q) for f in calls]
    loud = q.clone()
    loud[2, 0] *= times
    others = torch.ones(8, 2 * each, dtype=torch.bool, device="cuda")
    others[2, 0] = False
    for f, w in zip(calls, want):
        assert torch.equal(f(loud)[others], w[others])
    if group > 1:                                                          # pages that only row 2 holds
        mine = [p for p in rows[2] if not any(p in m for i, m in enumerate(rows) if i != 2)]
        assert mine
        if held == I8:
            pages.k_scale.view(n_pages, -1)[mine] *= times
            pages.v_scale.view(n_pages, -1)[mine] *= times
        else:
            pages.k.view(n_pages, -1)[mine] *= times
        others = torch.arange(8, device="cuda") != 2
        for f, w in zip(calls, want):
            assert torch.equal(f(q)[others], w[others])


@pytest.mark.parametrize("dtype,held", TYPES)
@pytest.mark.parametrize("page,kv,each,dim,group", [(16, 2, 3, 64, 1), (64, 4, 1, 128, 1), (16, 2, 4, 128, 4), (32, 1, 8, 64, 8), (256, 3, 7, 128, 2)])
def test_rows_over_pools_without_anything_spoiled(dtype, held, page, kv, each, dim, group):
    """The tests above have NaN wherever no row looks, with which sums are formed again; here none are."""
    lengths = [1, 0, 15, 16, 17, 33, page - 1, page, page + 1, 2 * page, 700, 129, 650, 300, 31, 5]
    check_attention(page + dim, lengths, page, kv, each, dim, dtype, held, group, 0.7, spoil=False)


@pytest.mark.parametrize("dtype,held", TYPES)
@pytest.mark.parametrize("group,spoil", [(1, False), (4, False), (1, True), (4, True)])
def test_results_in_the_place_of_the_queries(group, spoil, dtype, held):
    """... also where a value that is not finite has sums formed again, from the queries."""
    r = np.random.default_rng(3)
    lengths = [700, 33, 120, 650, 5, 0, 16, 300]
    rows, n_pages, stride = random_rows(r, lengths, 16, group, 0.7)
    pages, _ = pool_of(3, n_pages, 16, 2, 128, held)
    if spoil and held != I8:
        for i, n in enumerate(lengths):
            if n:
                pages.v.view(n_pages, 2, 16, 128)[rows[i][0], :, 3, 7] = math.inf
    table = table_of(rows, lengths, stride, 16, n_pages)
    q = randn(gen(1), 8, 10, 128, dtype=dtype)
    for most in (700, 1):
        want, place = ss.ss_attention_pages(q, pages, table, most, group), q.clone()
        assert ss.ss_attention_pages(place, pages, table, most, group, out=place) is place
        assert torch.equal(place, want) or (spoil and torch.equal(place.nan_to_num(), want.nan_to_num()))


@pytest.mark.parametrize("held", [F16, I8])
def test_pages_beyond_32_bits(held):
    """A pool of more than 2^32 bytes of keys; the rows' pages are its last ones."""
    n_pages, page, kv, dim = (9000 if held == F16 else 18000), 256, 8, 128
    pages = ss.Pages.allocate(n_pages, page, kv, dim, held)
    small, (k, v) = pool_of(2, 4, page, kv, dim, held)
    last = n_pages - 4
    for big, little in zip(pages.tensors, small.tensors):
        if big is not None:
            big.view(n_pages, -1)[last:] = little.view(4, -1)
    table = table_of([[last + 2, last], [last + 3]], [300, 256], 2, page, n_pages)
    q = randn(gen(1), 2, 8, dim, dtype=F16)
    got = ss.ss_attention_pages(q, pages, table, 300)
    low = ss.ss_attention_pages(q, small, table_of([[2, 0], [3]], [300, 256], 2, page, 4), 300)
    assert torch.equal(got, low) and low.any()
    rk, rv = ss.ss_pages_read(pages, table, i32([0, 1]), i32([299, 0]), F16)
    assert torch.equal(rk.double(), torch.stack([k[0, :, 43], k[3, :, 0]]).to(F16).double())
    ss.ss_pages_copy([pages], i32([last + 3]), i32([1]))
    assert torch.equal(pages.v.view(n_pages, -1)[1], pages.v.view(n_pages, -1)[last + 3])
    ss.ss_pages_copy([pages], i32([1]), i32([last + 1]))
    assert torch.equal(pages.k.view(n_pages, -1)[last + 1], small.k.view(4, -1)[3])


# ------------------------------------------------------------------------------------------------ fork
def plain_fork(table, lengths, page, n_pages, stride, parent, grow, held):
    """One row and one page at a time."""
    n_out, entries = len(parent), len(table[0]) if len(table) else 0
    rows, old, new = [], [], []
    for i, p in enumerate(parent):
        there = 0 <= p < len(table)
        a = min(max(lengths[p], 0), entries * page, stride * page) if there else 0
        more = (1 if there else 0) if grow is None else max(grow[i], 0)
        old.append(a)
        new.append(min(a + more, stride * page))
        rows.append([x if 0 <= x < n_pages else -1 for x in (table[p][:-(-a // page)] if there else [])])
    users, writers = {}, {}
    for i, r in enumerate(rows):
        for e, x in enumerate(r):
            if new[i] > old[i] and old[i] % page and e == len(r) - 1:
                writers.setdefault(x, []).append(i)
            else:
                users[x] = 1
    for x in range(n_pages):
        if held is not None and held[x]:
            users[x] = 1
    free = [x for x in range(n_pages) if x not in users and x not in writers]
    src, dst, missing, at = [-1] * n_out, [-1] * n_out, 0, 0
    def take():
        nonlocal at, missing
        at += 1
        if at <= len(free):
            return free[at - 1]
        missing += 1
        return -1
    for i, r in enumerate(rows):
        if new[i] > old[i] and old[i] % page and r and r[-1] >= 0:
            x = r[-1]
            if x in users or min(writers[x]) != i:
                r[-1] = take()
                if r[-1] >= 0:
                    src[i], dst[i] = x, r[-1]
        while len(r) < -(-new[i] // page):
            r.append(take())
    return [r + [-1] * (stride - len(r)) for r in rows], new, src, dst, missing


def check_fork(table, lengths, page, n_pages, stride, parent, grow=None, held=None, parents_given=True):
    n = len(parent)
    tb = table_of(table, lengths, len(table[0]) if len(table) else 0, page, n_pages)
    to = ss.PageTable(torch.full((n, stride), 77, dtype=torch.int32, device="cuda"), i32([55] * n), page, n_pages)
    before = [x.clone() for x in tb.tensors]
    kw = dict(parent=i32(parent) if parents_given else None, grow=None if grow is None else i32(grow),
              held=None if held is None else torch.tensor(held, dtype=torch.uint8, device="cuda"))
    src, dst, missing = ss.ss_pages_fork(tb, to, **kw)
    rows, new, a, b, m = plain_fork(table, lengths, page, n_pages, stride, parent, grow, held)
    assert to.lengths.tolist() == new
    assert to.pages.tolist() == rows
    assert (src.tolist(), dst.tolist(), missing.tolist()) == (a, b, [m])
    assert all(torch.equal(x, y) for x, y in zip(before, tb.tensors))
    return to, src, dst, missing


def random_table(r, n_rows, stride, page, n_pages):
    """Rows whose pages are their own, or in part another row's."""
    free, rows, lengths = list(r.permutation(n_pages)), [], []
    for i in range(n_rows):
        need = int(r.integers(0, stride + 1))
        share = int(r.integers(0, need + 1)) if i and r.random() < 0.6 else 0
        mine = list(rows[int(r.integers(i))][:share]) if share else []
        while len(mine) < need and free:
            mine.append(int(free.pop()))
        n = len(mine) * page - int(r.choice([0, 0, 1, 5, page - 1])) if mine else 0
        rows.append(mine + [-1] * (stride - len(mine)))
        lengths.append(max(n, 0))
    return rows, lengths


@pytest.mark.parametrize("seed", range(12))
@pytest.mark.parametrize("page", [16, 128])
def test_forks_of_random_tables(seed, page):
    r = np.random.default_rng(seed)
    n_in, stride = int(r.integers(1, 40)), int(r.integers(1, 12))
    n_pages = int(r.integers(n_in, n_in * stride * 2 + 2))
    table, lengths = random_table(r, n_in, stride, page, n_pages)
    n = int(r.integers(1, 60))
    parent = [int(x) for x in r.integers(-1, n_in + 1, n)]
    grow = None if seed % 3 == 0 else [int(x) for x in r.integers(-2, 2 * page, n)]
    held = None if seed % 2 else [int(x) for x in r.random(n_pages) < 0.1]
    check_fork(table, lengths, page, n_pages, max(stride + int(r.integers(-2, 4)), 1), parent, grow, held)


def test_what_a_fork_does():
    table, lengths = [[4, 6], [2, -1], [9, 3]], [20, 16, 32]
    # two children of a row in the middle of a page: the first keeps it, the second gets a copy; full pages are shared
    to, src, dst, _ = check_fork(table, lengths, 16, 12, 3, [0, 0, 1, 2])
    assert to.pages.tolist() == [[4, 6, -1], [4, 0, -1], [2, 1, -1], [9, 3, 5]] and src.tolist() == [-1, 6, -1, -1] and dst.tolist() == [-1, 0, -1, -1]
    check_fork(table, lengths, 16, 12, 3, [0, 1, 2], parents_given=False)          # rows go on as they are
    check_fork(table, lengths, 16, 12, 3, [0, 0, 0], grow=[0, 1, 1])               # one that stays: both others get copies
    check_fork(table, lengths, 16, 12, 3, [0, 0], grow=[0, 0])                     # all stay: none
    check_fork(table, lengths, 16, 12, 3, [0, -1, 1], grow=[3, 40, 16])            # a new row beside two old ones
    check_fork(table, lengths, 16, 12, 3, [0], held=[int(i == 6) for i in range(12)])
    check_fork(table, lengths, 16, 12, 2, [2, 1], grow=[10, 100])                  # no entries left
    check_fork(table, lengths, 16, 12, 1, [0, 1])                                  # fewer than the parent had
    check_fork([[0, 1]], [17], 16, 2, 2, [0, 0, 0])                                # a copy without a page for it
    check_fork([[0, 1]], [32], 16, 3, 4, [0, 0, -1], grow=[16, 17, 40])            # too few pages
    check_fork([[5, -3], [5, 1]], [30, 30], 16, 4, 2, [0, 1, 0])                   # entries that are no page
    check_fork([[-1], [-1]], [0, 0], 16, 1, 1, [0, 1, 1], grow=[1, 1, 1])
    check_fork([[1, 1]], [20], 16, 5, 3, [0])                                      # the same page twice


@pytest.mark.parametrize("n_pages,n", [(40000, 700), (5000, 3000), (4096, 1), (4097, 1025), (100003, 50), (16384, 1024), (16385, 1000), (16383, 900), (16384, 1000)])
def test_large_forks(n_pages, n):
    r = np.random.default_rng(n)
    table, lengths = random_table(r, 200, 20, 16, n_pages)
    check_fork(table, lengths, 16, n_pages, 24, [int(x) for x in r.integers(-1, 200, n)], [int(x) for x in r.integers(0, 60, n)])


@pytest.mark.parametrize("n_pages", [5, 20000])
def test_tables_of_nothing(n_pages):
    for rows, stride in ((0, 3), (3, 0), (0, 0)):
        a, b = (ss.PageTable.allocate(rows, stride, 16, n_pages) for _ in range(2))
        src, dst, missing = ss.ss_pages_fork(a, b)
        assert missing.item() == 0 and src.tolist() == dst.tolist() == [-1] * rows and b.lengths.tolist() == [0] * rows
        _, _, place, counts = ss.ss_pages_compact(a, b)
        assert counts.tolist() == [0, 0] and (place == -1).all()
        pages = ss.Pages.allocate(n_pages, 16, 1, 64, F16)
        q = randn(gen(1), rows, 2, 64, dtype=F16)
        assert not ss.ss_attention_pages(q, pages, a, 100).any()
        k = torch.ones(rows, 1, 64, dtype=F16, device="cuda")
        ss.ss_pages_write(pages, a, k, k)
        assert not pages.k.any()
        one = ss.PageTable.allocate(1, 2, 16, n_pages)
        ss.ss_pages_fork(a, one, i32([0]), i32([20]))
        assert one.pages.tolist() == [[0, 1]] and one.lengths.tolist() == [20]


def test_the_largest_number_of_rows():
    n = ss.SS_PAGES_MAX_ROWS
    check_fork([[0], [1]], [16, 3], 16, 20000, 2, [i % 3 for i in range(n)], None)


# ------------------------------------------------------------------------------------------------ compact
def check_compact(table, lengths, page, n_pages, held=None, in_place=False):
    stride = len(table[0])
    tb = table_of(table, lengths, stride, page, n_pages)
    to = None if in_place else ss.PageTable(torch.full((len(table), stride), 77, dtype=torch.int32, device="cuda"), i32([5] * len(table)), page, n_pages)
    src, dst, place, counts = ss.ss_pages_compact(tb, to, None if held is None else torch.tensor(held, dtype=torch.uint8, device="cuda"))
    got = tb if in_place else to
    cut = [[x if 0 <= x < n_pages and e * page < n else -1 for e, x in enumerate(r)] for r, n in zip(table, lengths)]
    used = sorted({x for r in cut for x in r if x >= 0} | {x for x in range(n_pages) if held and held[x]})
    high = [x for x in used if x >= len(used)]
    holes = [x for x in range(len(used)) if x not in set(used)]
    new = {x: x for x in used}
    new.update(zip(high, holes))
    assert counts.tolist() == [len(used), len(high)]
    assert src.tolist() == high + [-1] * (n_pages // 2 - len(high)) and dst.tolist() == holes + [-1] * (n_pages // 2 - len(high))
    assert place.tolist() == [new.get(x, -1) for x in range(n_pages)]
    assert got.pages.tolist() == [[new[x] if x >= 0 else -1 for x in r] for r in cut]
    assert got.lengths.tolist() == [min(max(n, 0), stride * page) for n in lengths]
    return tb, src, dst, counts


@pytest.mark.parametrize("seed", range(8))
@pytest.mark.parametrize("in_place", [False, True])
def test_random_tables_become_dense(seed, in_place):
    r = np.random.default_rng(seed)
    n_rows, stride = int(r.integers(1, 30)), int(r.integers(1, 12))
    n_pages = int(r.integers(1, n_rows * stride * 3 + 2))
    table, lengths = random_table(r, n_rows, stride, 16, n_pages)
    check_compact(table, lengths, 16, n_pages, None if seed % 2 else [int(x) for x in r.random(n_pages) < 0.1], in_place)


def test_dense_empty_and_large_pools():
    check_compact([[0, 1], [2, -1]], [32, 3], 16, 5)
    check_compact([[-1, 9], [7, 2]], [32, -4], 16, 5)
    check_compact([[0]], [1], 16, 1)
    check_compact([[4]], [16], 16, 5, in_place=True)
    r = np.random.default_rng(1)
    check_compact(*random_table(r, 300, 60, 16, 50001), 16, 50001)
    check_compact(*random_table(r, 30, 60, 16, 4096), 16, 4096)
    for n in (8191, 8192, 8193, 16384):
        check_compact(*random_table(r, 200, 60, 16, n), 16, n)
        check_compact(*random_table(r, 500, 20, 16, n), 16, n, in_place=True)


# ------------------------------------------------------------------------------------------------ copies
@pytest.mark.parametrize("held", [F16, I8])
@pytest.mark.parametrize("n_layers,page,kv,dim", [(1, 16, 1, 64), (3, 32, 5, 128), (33, 16, 2, 64), (70, 256, 1, 64)])
def test_pages_are_copied_in_every_layer(held, n_layers, page, kv, dim):
    n_pages = 40
    layers = [pool_of(i, n_pages, page, kv, dim, held)[0] for i in range(n_layers)]
    before = [[None if x is None else x.clone() for x in layer.tensors] for layer in layers]
    src = [3, -1, 5, 39, 5, 7, 40, 2, 2**31 - 1, 8]
    dst = [0, 9, 11, 38, 12, -1, 13, 40, 14, 8]
    ss.ss_pages_copy(layers, i32(src), i32(dst))
    for layer, old in zip(layers, before):
        for x, y in zip(layer.tensors, old):
            if x is None:
                continue
            want = y.view(n_pages, -1).clone()
            for a, b in ((3, 0), (5, 11), (39, 38), (5, 12)):
                want[b] = y.view(n_pages, -1)[a]
            assert torch.equal(x.view(n_pages, -1), want)


@pytest.mark.parametrize("count", [0, 1, 5, 9000, -3, 20000])
def test_as_many_pairs_as_the_device_says(count):
    n_pages, n = 20000, 9000
    layer = pool_of(1, n_pages, 16, 1, 64, F16)[0]
    old = layer.k.view(n_pages, -1).clone()
    order = torch.randperm(n_pages, device="cuda", generator=gen(2)).int()
    src, dst = order[:n].contiguous(), order[n:2 * n].contiguous()
    ss.ss_pages_copy([layer], src, dst, i32([count]))
    k = min(max(count, 0), n)
    old[dst[:k].long()] = old[src[:k].long()]
    assert torch.equal(layer.k.view(n_pages, -1), old)


# ------------------------------------------------------------------------------------------------ streams, graphs, a run of them
@pytest.mark.parametrize("group", [1, 4])
def test_the_same_call_gives_the_same_bits_in_graphs_and_on_streams(group):
    r = np.random.default_rng(0)
    lengths = [int(x) for x in r.integers(500, 3000, 16)]
    rows, n_pages, stride = random_rows(r, lengths, 16, group, 0.8)
    pages, _ = pool_of(0, n_pages + 40, 16, 4, 128, I8)
    table = table_of(rows, lengths, stride, 16, n_pages + 40)
    to = ss.PageTable.allocate(16, stride, 16, n_pages + 40)
    q, k, v = randn(gen(1), 16, 16, 128, dtype=F16), randn(gen(2), 16, 4, 128, dtype=F16), randn(gen(3), 16, 4, 128, dtype=F16)
    parent = i32([i // group * group + int(x) for i, x in enumerate(r.integers(0, group, 16))])

    def step():
        src, dst, missing = ss.ss_pages_fork(table, to, parent)
        ss.ss_pages_copy([pages], src, dst)
        ss.ss_pages_write(pages, to, k, v)
        return ss.ss_attention_pages(q, pages, to, 3001, group), to.pages.clone(), src, missing

    first = step()
    assert first[3].item() == 0
    for x, y in zip(first, step()):
        assert torch.equal(x, y)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = step()
    torch.cuda.current_stream().wait_stream(other)
    for x, y in zip(first, got):
        assert torch.equal(x, y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = step()
    for _ in range(3):
        to.pages.fill_(-1)
        g.replay()
        torch.cuda.synchronize()
        assert (ss.ss_attention_pages(q, pages, to, 3001, group) - held[0]).abs().max() == 0
        for x, y in zip(first, held):
            assert torch.equal(x, y)


def test_a_given_stream_is_ordered_behind_the_current_one():
    pages, _ = pool_of(0, 9, 16, 2, 64, F16)
    table = table_of([[1, 2], [3, 4]], [30, 20], 3, 16, 9)
    q = randn(gen(1), 2, 2, 64, dtype=F16)
    want = ss.ss_attention_pages(q, pages, table, 30)
    s = torch.cuda.Stream()
    q2 = torch.zeros_like(q)
    torch.cuda._sleep(20_000_000)
    q2.copy_(q)
    got = ss.ss_attention_pages(q2, pages, table, 30, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(got, want)

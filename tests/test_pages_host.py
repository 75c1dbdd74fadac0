"""What the operators on caches in pages and of beam search refuse.  No GPU is touched: the pointers lead nowhere, and every call is refused, or has
nothing to do, before it would launch."""
import ctypes as C

import pytest
import torch

from paper_2305_13144_amd import binding as ss
from test_operators_host import BAD_ROWS, P, lib, refused, rows  # noqa: F401

Q = 2 * P


def pages(**kw):
    d = dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=10, page_slots=16, n_kv_heads=2, head_dim=64, dtype=ss.SS_I8)
    d.update(kw)
    return ss.ss_pages(*d.values())


def table(**kw):
    d = dict(pages=P, lengths=P, n_rows=8, stride=4, page_slots=16, n_pages=10)
    d.update(kw)
    return ss.ss_page_table(*d.values())


def beams(**kw):
    d = dict(totals=P, lengths=P, ended=P, history=None, history_stride=0)
    d.update(kw)
    return ss.ss_beams(*d.values())


def write(lib, p=pages(), t=table(), k=rows(), v=rows(), row=P, pos=P, n=8):
    return lib.ss_pages_write(p, t, k, v, row, pos, n, None)


def read(lib, p=pages(), t=table(), k=rows(), v=rows(), row=P, pos=P, n=8):
    return lib.ss_pages_read(p, t, row, pos, n, k, v, None)


def attend(lib, p=pages(), t=table(), q=rows(), out=rows(), heads=4, n=8, rows=None, most=64, group=1, scale=0.1, work=P, nbytes=1 << 40):
    return lib.ss_attention_pages(p, t, q, out, heads, n, rows, most, group, scale, work, nbytes, None)


def fork(lib, a=table(), b=table(pages=Q, lengths=Q), parent=P, grow=P, held=P, src=P, dst=P, missing=P, work=P, nbytes=80):
    return lib.ss_pages_fork(a, b, parent, grow, held, src, dst, missing, work, nbytes, None)


def compact(lib, a=table(), b=table(pages=Q, lengths=Q), held=P, src=P, dst=P, place=P, counts=P, work=P, nbytes=80):
    return lib.ss_pages_compact(a, b, held, src, dst, place, counts, work, nbytes, None)


def copy(lib, layers=(pages(),), src=P, dst=P, n=4, count=None):
    return lib.ss_pages_copy((ss.ss_pages * len(layers))(*layers), len(layers), src, dst, n, count, None)


def select(lib, logits=P, dtype=ss.SS_F32, stride=100, groups=2, n=3, vocab=100, keep=4, now=beams(), next=beams(totals=Q, lengths=Q, ended=Q), parent=P,
           token=P, end=7, power=0.5, work=P, nbytes=1 << 40):
    return lib.ss_beam_select(logits, dtype, stride, groups, n, vocab, keep, now, next, parent, token, end, power, work, nbytes, None)


BAD_PAGES = [(None, "NULL"), (pages(head_dim=96), "head_dim"), (pages(dtype=ss.SS_F32), "dtype"), (pages(n_kv_heads=0), "heads"), (pages(n_kv_heads=65536), "heads"),
             (pages(n_pages=0), "page"), (pages(n_pages=-1), "page"), (pages(page_slots=8), "page_slots"), (pages(page_slots=48), "page_slots"),
             (pages(page_slots=512), "page_slots"), (pages(k=0), "NULL"), (pages(v=P + 8), "aligned"), (pages(v_scale=0), "k_scale"), (pages(k_scale=P + 4), "aligned")]
BAD_TABLES = [(None, "NULL"), (table(n_rows=-1), "negative"), (table(stride=-1), "negative"), (table(n_pages=0), "page"), (table(page_slots=24), "page_slots"),
              (table(lengths=0), "NULL"), (table(pages=0), "NULL"), (table(stride=2**27), "positions"), (table(n_rows=2**20, stride=2**12), "entries")]


@pytest.mark.parametrize("p,word", BAD_PAGES)
def test_bad_pages_are_refused(lib, p, word):
    for call in (write, read, attend):
        refused(call(lib, p=p), word)
    if p is not None:
        refused(copy(lib, layers=(p,)), word)
        refused(copy(lib, layers=(pages(), p)), word)


@pytest.mark.parametrize("t,word", BAD_TABLES)
def test_bad_tables_are_refused(lib, t, word):
    for call in (write, read, attend):
        refused(call(lib, t=t), word)
    for call in (fork, compact):
        refused(call(lib, a=t), word)
        refused(call(lib, b=t), word)


@pytest.mark.parametrize("r,word", BAD_ROWS)
def test_bad_rows_are_refused(lib, r, word):
    for call, names in ((write, "kv"), (read, "kv"), (attend, ("q", "out"))):
        for name in names:
            refused(call(lib, **{name: r}), word)


def test_tokens_that_do_not_fit_are_refused(lib):
    for call in (write, read):
        for other in (table(page_slots=32), table(n_pages=11)):
            refused(call(lib, t=other), "differ")
        refused(call(lib, n=-1), "negative")
        refused(call(lib, n=9), "fewer")
        refused(call(lib, row=None), "together")
        refused(call(lib, pos=None), "together")
        refused(call(lib, v=rows(dtype=ss.SS_BF16)), "type")
        wide = rows(row_stride=0 if call is write else 2**20, rows=2**31 - 1)
        refused(call(lib, k=wide, v=wide, n=2**28), "tokens")
        refused(call(lib, p=pages(n_kv_heads=9), k=wide, v=wide, n=2**28 - 16), "vectors")
        assert call(lib, n=0) == ss.SS_OK
        assert call(lib, t=table(n_rows=0, lengths=0, pages=0)) == ss.SS_OK
        assert call(lib, t=table(stride=0, pages=0)) == ss.SS_OK
    refused(read(lib, k=rows(row_stride=64)), "overlap")
    refused(read(lib, v=rows(row_stride=0)), "overlap")


def test_attention_that_does_not_fit_is_refused(lib):
    refused(attend(lib, t=table(page_slots=32)), "differ")
    refused(attend(lib, t=table(n_pages=9)), "differ")
    refused(attend(lib, heads=3), "multiple")
    refused(attend(lib, heads=0), "multiple")
    refused(attend(lib, heads=65536), "heads")
    refused(attend(lib, n=-1), "negative")
    refused(attend(lib, most=-1), "negative")
    refused(attend(lib, n=65536), "65535")
    refused(attend(lib, n=9, rows=P), "fewer")
    many = rows(rows=65535, row_stride=2**20)
    refused(attend(lib, n=65535, rows=P, q=many, out=many, p=pages(n_kv_heads=65), heads=65), "too many")
    refused(attend(lib, t=table(n_rows=7)), "table has fewer")
    refused(attend(lib, out=rows(rows=7)), "fewer")
    refused(attend(lib, out=rows(dtype=ss.SS_BF16)), "type")
    refused(attend(lib, p=pages(dtype=ss.SS_BF16)), "type")
    refused(attend(lib, out=rows(row_stride=0)), "overlap")
    for group in (0, -1, 33):
        refused(attend(lib, group=group), "group")
    refused(attend(lib, group=3), "whole groups")
    for scale in (float("nan"), float("inf")):
        refused(attend(lib, scale=scale), "finite")
    assert attend(lib, n=0) == ss.SS_OK
    need = C.c_size_t(0)
    assert lib.ss_attention_pages_workspace(4, 2, 64, 16, 4, 8, 64, 2, need) == ss.SS_OK
    for bad, word in (((4, 3, 64, 16, 4, 8, 64, 2), "multiple"), ((4, 2, 65, 16, 4, 8, 64, 2), "head_dim"), ((4, 2, 64, 17, 4, 8, 64, 2), "page_slots"),
                      ((4, 2, 64, 16, -1, 8, 64, 2), "length"), ((4, 2, 64, 256, 2**23, 8, 64, 2), "positions"), ((4, 2, 64, 16, 4, 9, 64, 2), "whole"),
                      ((4, 2, 64, 16, 4, 8, 64, 0), "group"), ((4, 2, 64, 16, 4, 8, -64, 1), "negative")):
        refused(lib.ss_attention_pages_workspace(*bad, need), word)
    refused(lib.ss_attention_pages_workspace(4, 2, 64, 16, 4, 8, 64, 2, None), "NULL")


def test_a_workspace_of_the_attention_that_is_too_small_is_refused_with_its_size(lib):
    need = C.c_size_t(0)
    assert lib.ss_attention_pages_workspace(4, 2, 64, 16, 4000, 8, 64000, 4, need) == ss.SS_OK
    if need.value == 0:
        pytest.skip("these counts take no workspace")
    t = table(stride=4000)
    for work, n in ((None, 0), (P, need.value - 1), (None, need.value)):
        refused(attend(lib, t=t, most=64000, group=4, work=work, nbytes=n), str(need.value))
    refused(attend(lib, t=t, most=64000, group=4, work=P + 4, nbytes=need.value), "aligned")


def test_a_longest_length_beyond_the_entries_shares_out_as_the_entries_do(lib):
    """No row is longer than its entries: what a caller allows beyond that takes no workspace (and no time)."""
    a, b = C.c_size_t(0), C.c_size_t(0)
    for stride, n, group in ((4, 65535, 1), (60, 16384, 8), (800, 40, 1), (3000, 16, 4), (0, 5, 5)):
        assert lib.ss_attention_pages_workspace(4, 1, 128, 64, stride, n, 64 * stride, group, a) == ss.SS_OK
        assert lib.ss_attention_pages_workspace(4, 1, 128, 64, stride, n, 2**31 - 1, group, b) == ss.SS_OK
        assert a.value == b.value


def test_forks_and_compactions_that_do_not_fit_are_refused(lib):
    for call in (fork, compact):
        for other in (table(pages=Q, lengths=Q, page_slots=32), table(pages=Q, lengths=Q, n_pages=9)):
            refused(call(lib, b=other), "differ")
        many = ss.SS_PAGES_MAX_ROWS + 1
        refused(call(lib, a=table(n_rows=many), b=table(pages=Q, lengths=Q, n_rows=many)), "rows")
        refused(call(lib, src=None), "NULL")
        refused(call(lib, dst=None), "NULL")
        refused(call(lib, work=None), "80")
        refused(call(lib, nbytes=79), "80")
        refused(call(lib, work=P + 8), "aligned")
    refused(fork(lib, missing=None), "NULL")
    refused(fork(lib, b=table(lengths=Q)), "must not be")
    refused(fork(lib, b=table(pages=Q)), "must not be")
    refused(compact(lib, counts=None), "NULL")
    refused(compact(lib, b=table(pages=Q, lengths=Q, n_rows=7)), "rows or stride")
    refused(compact(lib, b=table(pages=Q, lengths=Q, stride=3)), "rows or stride")
    need = C.c_size_t(0)
    assert lib.ss_pages_workspace(10, need) == ss.SS_OK and need.value == 80
    refused(lib.ss_pages_workspace(0, need), "page")
    refused(lib.ss_pages_workspace(5, None), "NULL")


@pytest.mark.parametrize("n", [ss.SS_PAGES_MAX + 1, 2**31 - 1])
def test_more_pages_than_any_pool_has_are_refused(lib, n):
    """Where pages are counted, sums of their numbers and of a step of 4 x 4096 are 32 bits."""
    a, b, p = table(n_pages=n), table(pages=Q, lengths=Q, n_pages=n), pages(n_pages=n)
    for call in (fork, compact):
        refused(call(lib, a=a, b=b, nbytes=1 << 40), "at most")
    for call in (write, read, attend):
        refused(call(lib, p=p, t=a), "at most")
    refused(copy(lib, layers=(p,)), "at most")
    need = C.c_size_t(0)
    refused(lib.ss_pages_workspace(n, need), "at most")
    assert lib.ss_pages_workspace(ss.SS_PAGES_MAX, need) == ss.SS_OK and need.value == 8 * ss.SS_PAGES_MAX


def test_groups_whose_pieces_pass_32_bits_are_refused(lib):
    """A group's list of pieces of 16 positions is counted in 32 bits; its rows may have nothing in common."""
    need = C.c_size_t(0)
    for page, stride in ((16, 2**26), (256, 2**22)):                   # 2^30 positions a row, 32 rows: 2^31 pieces
        refused(lib.ss_attention_pages_workspace(4, 2, 64, page, stride, 32, 64, 32, need), "pieces")
        refused(attend(lib, p=pages(page_slots=page), t=table(page_slots=page, stride=stride, n_rows=1), rows=P, q=rows(rows=32), out=rows(rows=32), n=32, group=32),
                "pieces")
        assert lib.ss_attention_pages_workspace(4, 2, 64, page, stride - 1, 32, 64, 32, need) == ss.SS_OK
        assert lib.ss_attention_pages_workspace(4, 2, 64, page, stride, 32, 64, 1, need) == ss.SS_OK


def test_tables_that_lie_in_each_other_are_refused(lib):
    """Tables of 8 rows of 4 entries, 128 bytes, and 8 lengths, 32: what is written where the other table is read could lead out of it."""
    for call, word in ((fork, "share memory"), (compact, "share no memory")):
        for at in (P - 124, P - 4, P + 4, P + 124):
            refused(call(lib, b=table(pages=at, lengths=Q)), word)
        for at in (P - 28, P + 4, P + 124):                            # its lengths among the other's entries
            refused(call(lib, a=table(lengths=Q), b=table(pages=2 * Q, lengths=at)), word)
            refused(call(lib, a=table(pages=2 * Q, lengths=at), b=table(lengths=Q)), word)
        refused(call(lib, a=table(pages=2 * Q), b=table(pages=3 * Q, lengths=P + 28)), word)


def test_copies_that_do_not_fit_are_refused(lib):
    for other in (pages(n_pages=11), pages(page_slots=32), pages(n_kv_heads=1), pages(head_dim=128), pages(dtype=ss.SS_F16)):
        refused(copy(lib, layers=(pages(), other)), "layer 1")
    refused(copy(lib, src=None), "NULL")
    refused(copy(lib, dst=None), "NULL")
    refused(copy(lib, n=-1), "negative")
    refused(lib.ss_pages_copy(None, -1, P, P, 1, None, None), "negative")
    refused(lib.ss_pages_copy(None, 1, P, P, 1, None, None), "layers is NULL")
    assert copy(lib, n=0, src=None, dst=None) == ss.SS_OK
    assert lib.ss_pages_copy(None, 0, P, P, 1, None, None) == ss.SS_OK


def test_steps_of_beam_search_that_do_not_fit_are_refused(lib):
    refused(select(lib, n=0), "beams")
    refused(select(lib, n=65), "beams")
    refused(select(lib, keep=0), "keep")
    refused(select(lib, keep=65), "keep")
    refused(select(lib, vocab=0, end=-1), "vocab")
    refused(select(lib, groups=-1), "rows")
    refused(select(lib, groups=65535, n=2), "rows")
    refused(select(lib, dtype=ss.SS_I8), "dtype")
    refused(select(lib, now=None), "NULL")
    refused(select(lib, next=None), "NULL")
    refused(select(lib, logits=None), "NULL")
    refused(select(lib, parent=None), "NULL")
    refused(select(lib, token=None), "NULL")
    refused(select(lib, now=beams(totals=0)), "NULL")
    refused(select(lib, next=beams(totals=0, lengths=Q, ended=Q)), "NULL")
    refused(select(lib, logits=P + 2), "aligned")
    refused(select(lib, logits=P + 1, dtype=ss.SS_BF16), "aligned")
    refused(select(lib, stride=-1), "row_stride")
    refused(select(lib, stride=2**41), "row_stride")
    for end in (-2, 100):
        refused(select(lib, end=end), "end_id")
    for power in (float("nan"), float("inf")):
        refused(select(lib, power=power), "finite")
    refused(select(lib, now=beams(lengths=0)), "lengths")
    refused(select(lib, now=beams(lengths=0), power=0.0), "lengths")
    refused(select(lib, now=beams(history=P, history_stride=4)), "both")
    refused(select(lib, now=beams(history=P, history_stride=-4), next=beams(totals=Q, lengths=Q, ended=Q, history=Q, history_stride=4)), "history_stride")
    for same in (beams(lengths=Q, ended=Q), beams(totals=Q, ended=Q), beams(totals=Q, lengths=Q)):
        refused(select(lib, next=same), "must not be")
    need = C.c_size_t(0)
    assert lib.ss_beam_select_workspace(2, 3, 100, 4, need) == ss.SS_OK and need.value > 0
    refused(select(lib, work=None), str(need.value))
    refused(select(lib, nbytes=need.value - 1), str(need.value))
    refused(select(lib, work=P + 4), "aligned")
    refused(lib.ss_beam_select_workspace(2, 3, 100, 4, None), "NULL")
    refused(lib.ss_beam_select_workspace(2, 3, 100, 65, need), "keep")
    assert select(lib, groups=0) == ss.SS_OK


def test_tensors_and_numbers_that_do_not_fit_are_refused_by_the_binding(lib):
    half, ints = torch.zeros(2048, dtype=torch.float16), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        ss.Pages(half, half, 16, 1, 64)
    with pytest.raises(ValueError, match="GPU"):
        ss.PageTable(ints.view(2, 2), torch.zeros(2, dtype=torch.int32), 16, 4)
    with pytest.raises(ValueError, match="GPU"):
        ss.ss_beam_select(torch.zeros(2, 8), torch.zeros(1, 2), 2)
    for bad in (dict(page_slots=20), dict(n_kv_heads=0), dict(head_dim=32)):
        with pytest.raises(ValueError):
            ss.Pages.allocate(**{**dict(n_pages=4, page_slots=16, n_kv_heads=1, head_dim=64, dtype=torch.int8, device="meta"), **bad})
    for n in (2**32 + 5, 2**31):
        for name in ("n_heads", "n_kv_heads", "stride", "n", "max_length", "group"):
            with pytest.raises(ValueError, match=name):
                ss.ss_attention_pages_workspace(**{**dict(n_heads=4, n_kv_heads=2, head_dim=64, page_slots=16, stride=4, n=8, max_length=9, group=1), name: n})
        for name in ("n_groups", "beams", "vocab", "keep"):
            with pytest.raises(ValueError, match=name):
                ss.ss_beam_select_workspace(**{**dict(n_groups=2, beams=2, vocab=9, keep=2), name: n})
        with pytest.raises(ValueError, match="n_pages"):
            ss.ss_pages_workspace(n)
    assert ss.ss_pages_workspace(7) == 56

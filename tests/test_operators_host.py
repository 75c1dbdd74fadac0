"""What the operators on device tensors refuse, the masks of trees, and the plan of the attention over a cache.  No GPU is touched:
the pointers lead nowhere, and every call is refused, or has nothing to do, before it would launch."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2305_13144_amd import binding as ss

P = 1 << 20   # an aligned address that nothing may follow


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(ss.LIB_PATH):
        from paper_2305_13144_amd import build
        build.build()
    return ss.lib()


def cache(**kw):
    d = dict(k=P, v=P, k_scale=P, v_scale=P, start=P, slots=P, total_slots=100, n_seq=4, n_kv_heads=2, head_dim=64, dtype=ss.SS_I8)
    d.update(kw)
    return ss.ss_cache(*d.values())


def rows(**kw):
    d = dict(p=P, row_stride=256, head_stride=64, rows=8, dtype=ss.SS_F16)
    d.update(kw)
    return ss.ss_rows(*d.values())


def refused(rc, word):
    assert rc == ss.SS_EINVAL
    assert word in ss.lib().ss_last_error().decode(), ss.lib().ss_last_error()


BAD_CACHES = [(None, "NULL"), (cache(head_dim=96), "head_dim"), (cache(dtype=ss.SS_F32), "dtype"), (cache(n_kv_heads=0), "heads"),
              (cache(n_seq=-1), "sequences"), (cache(k=0), "NULL"), (cache(v=P + 8), "aligned"), (cache(k_scale=0), "k_scale"),
              (cache(start=0), "start"), (cache(total_slots=-1), "slots")]
BAD_ROWS = [(None, "NULL"), (rows(p=0), "NULL"), (rows(p=P + 2), "aligned"), (rows(row_stride=100), "strides"),
            (rows(head_stride=4), "strides"), (rows(dtype=ss.SS_F32), "dtype"), (rows(dtype=ss.SS_I8), "dtype"), (rows(rows=-1), "rows")]


def write(lib, c=cache(), k=rows(), v=rows(), seq=P, slot=P, n=8):
    return lib.ss_cache_write(c, k, v, seq, slot, n, None)


def read(lib, c=cache(), k=rows(), v=rows(), seq=P, slot=P, n=8):
    return lib.ss_cache_read(c, seq, slot, n, k, v, None)


def tree(lib, c=cache(), q=rows(), out=rows(), heads=4, n_seq=4, seq=None, context=P, max_context=50, nodes=None, max_nodes=1, mask=None,
         work=None, nbytes=0, scale=0.1):
    return lib.ss_attention_tree(c, q, out, heads, n_seq, seq, context, max_context, nodes, max_nodes, mask, scale, work, nbytes, None)


def packed(lib, q=rows(), k=rows(), v=rows(), out=rows(), heads=4, kv=2, dim=64, offsets=P, n_seq=2, max_len=8, scale=0.1):
    return lib.ss_attention_packed(q, k, v, out, heads, kv, dim, offsets, n_seq, max_len, scale, None)


@pytest.mark.parametrize("c,word", BAD_CACHES)
def test_bad_caches_are_refused(lib, c, word):
    for call in (write, read, tree):
        refused(call(lib, c), word)


@pytest.mark.parametrize("r,word", BAD_ROWS)
def test_bad_rows_are_refused(lib, r, word):
    for call in (write, read, packed):
        for name in ("k", "v"):
            refused(call(lib, **{name: r}), word)
    for call in (tree, packed):
        for name in ("q", "out"):
            refused(call(lib, **{name: r}), word)


def test_calls_whose_parts_do_not_fit_are_refused(lib):
    for call in (write, read):
        refused(call(lib, n=-1), "negative")
        refused(call(lib, n=9), "rows")
        refused(call(lib, seq=None), "seq")
        refused(call(lib, slot=None), "slot")
        refused(call(lib, v=rows(dtype=ss.SS_BF16)), "type")
    refused(tree(lib, heads=3), "multiple")
    refused(tree(lib, heads=0), "multiple")
    refused(tree(lib, n_seq=-1), "negative")
    refused(tree(lib, max_context=-1), "negative")
    refused(tree(lib, max_context=2**31 - 1), "max_context")
    refused(tree(lib, max_nodes=0, nodes=P), "max_nodes")
    refused(tree(lib, max_nodes=1025, nodes=P), "max_nodes")
    refused(tree(lib, max_nodes=2), "nodes is NULL")
    refused(tree(lib, n_seq=5), "sequences")
    refused(tree(lib, seq=P, n_seq=9), "rows")
    refused(tree(lib, context=None), "context")
    refused(tree(lib, out=rows(rows=7)), "fewer rows")
    refused(tree(lib, out=rows(dtype=ss.SS_BF16)), "type")
    refused(tree(lib, c=cache(dtype=ss.SS_BF16)), "type")
    refused(tree(lib, seq=P, n_seq=65535, heads=64, q=rows(rows=2**40), out=rows(rows=2**40), nodes=P, max_nodes=1024), "too many")
    refused(tree(lib, seq=P, n_seq=65536, q=rows(rows=2**40), out=rows(rows=2**40)), "sequences")
    refused(tree(lib, c=cache(n_seq=0, start=0, slots=0), seq=P), "no sequences")
    refused(tree(lib, q=rows(row_stride=-64)), "strides")
    refused(tree(lib, q=rows(head_stride=2**60)), "strides")
    refused(packed(lib, heads=65536), "heads")
    refused(packed(lib, heads=5), "multiple")
    refused(packed(lib, dim=80), "head_dim")
    refused(packed(lib, k=rows(dtype=ss.SS_BF16)), "type")
    refused(packed(lib, v=rows(rows=7)), "fewer rows")
    refused(packed(lib, offsets=None), "offsets")
    refused(packed(lib, n_seq=-1), "negative")
    refused(packed(lib, max_len=-1), "negative")
    refused(packed(lib, n_seq=65536), "sequences")
    refused(packed(lib, max_len=1 << 30), "max_len")


def test_results_that_overlap_and_scales_that_are_no_numbers_are_refused(lib):
    for bad in (rows(row_stride=0), rows(head_stride=0), rows(row_stride=192, head_stride=64), rows(row_stride=64, head_stride=448), rows(head_stride=32)):
        refused(tree(lib, out=bad), "overlap")
        refused(packed(lib, out=bad), "overlap")
    for bad in (rows(row_stride=64), rows(head_stride=32), rows(row_stride=0)):
        refused(read(lib, k=bad), "overlap")
        refused(read(lib, v=bad), "overlap")
    for scale in (float("nan"), float("inf"), -float("inf")):
        refused(tree(lib, scale=scale), "finite")
        refused(packed(lib, scale=scale), "finite")
    by_heads = rows(row_stride=64, head_stride=512)                # [heads][rows]
    assert tree(lib, out=by_heads, n_seq=0, context=None) == ss.SS_OK and packed(lib, out=by_heads, n_seq=0) == ss.SS_OK


def test_a_workspace_that_is_too_small_is_refused_with_its_size(lib):
    need = C.c_size_t(0)
    assert lib.ss_attention_tree_workspace(4, 2, 64, 1, 50000, 1, need) == ss.SS_OK and need.value > 0
    for work, n in ((None, 0), (P, need.value - 1), (None, need.value)):
        refused(tree(lib, n_seq=1, max_context=50000, work=work, nbytes=n), str(need.value))
    refused(tree(lib, n_seq=1, max_context=50000, work=P + 4, nbytes=need.value), "aligned")
    refused(lib.ss_attention_tree_workspace(4, 2, 64, 1, 50000, 1, None), "NULL")
    refused(lib.ss_attention_tree_workspace(4, 2, 72, 1, 50000, 1, need), "head_dim")
    refused(lib.ss_attention_tree_workspace(4, 3, 64, 1, 50000, 1, need), "multiple")


def test_calls_of_nothing_have_nothing_to_do(lib):
    assert write(lib, n=0, seq=None, slot=None) == ss.SS_OK
    assert read(lib, n=0, seq=None, slot=None) == ss.SS_OK
    assert write(lib, c=cache(n_seq=0, total_slots=0, k=0, v=0, start=0, slots=0)) == ss.SS_OK
    assert tree(lib, n_seq=0, context=None) == ss.SS_OK
    assert packed(lib, n_seq=0) == ss.SS_OK
    assert packed(lib, max_len=0) == ss.SS_OK


def test_masks_of_trees(lib):
    parents = [-1, 0, 0, 2, -1, 4, 3] + list(range(6, 80))
    mask = ss.ss_tree_mask(parents, 100).view(np.uint64)
    for t in range(len(parents)):
        sees, u = set(), t
        while u >= 0:
            sees.add(u)
            u = parents[u]
        assert {b for b in range(128) if int(mask[t, b // 64]) >> (b % 64) & 1} == sees
    assert ss.ss_tree_mask([], 5).shape == (0, 1)
    for bad in ([0], [-1, 1], [-2], [-1, 5]):
        with pytest.raises(ss.SsError) as e:
            ss.ss_tree_mask(bad, 64)
        assert e.value.code == ss.SS_EINVAL
    for n, top in ((3, 2), (1, 0), (1, 1025)):
        with pytest.raises(ss.SsError):
            ss.ss_tree_mask([-1] * n, top)


def test_tensors_that_do_not_fit_are_refused_by_the_binding(lib):
    host = torch.zeros(4, 2, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="GPU"):
        ss.Cache(torch.zeros(256, dtype=torch.float16), torch.zeros(256, dtype=torch.float16), torch.zeros(1, dtype=torch.int64),
                 torch.zeros(1, dtype=torch.int32), 2, 64)
    with pytest.raises(ValueError, match="GPU"):
        ss.ss_attention_packed(host, host, host, torch.zeros(2, dtype=torch.int32), 4)


def test_rows_that_require_gradients_are_refused(lib):
    ss._with_torch()
    x = torch.zeros(4, 2, 64, dtype=torch.float16, requires_grad=True)
    with pytest.raises(ValueError, match="q requires gradients"):
        ss._rows(x, "q", -1, 2, 64)                                # -1: the host, where nothing is launched
    with pytest.raises(ValueError, match="gradients"):
        ss._rows((x * 2)[1:], "q", -1, 2, 64)
    with torch.no_grad():
        assert ss._rows(x, "q", -1, 2, 64).rows == 4
    assert ss._rows(x.detach(), "q", -1, None, 64).row_stride == 128


def test_more_tokens_than_a_launch_takes_are_refused(lib):
    """Rows of stride 0 let any number of tokens share a vector."""
    one, all_ = cache(n_kv_heads=1), rows(row_stride=0, rows=2**31 - 1)
    for n in (2**28 - 15, 2**28, 2**31 - 16, 2**31 - 1):
        refused(write(lib, c=one, k=all_, v=all_, n=n), "tokens")
        refused(read(lib, c=one, k=rows(rows=2**31 - 1), v=rows(rows=2**31 - 1), n=n), "tokens")
    nothing = cache(n_kv_heads=1, n_seq=0, start=0, slots=0)
    assert write(lib, c=nothing, k=all_, v=all_, n=2**28 - 16) == ss.SS_OK
    refused(write(lib, c=cache(n_kv_heads=9), k=all_, v=all_, n=2**28 - 16), "vectors")


def test_numbers_beyond_32_bits_are_refused_by_the_binding(lib):
    """2^32 + 5 would be 5 where the library takes 32 bits, and 2^31 slots none."""
    for n in (2**32 + 5, 2**31, -2**31 - 1):
        with pytest.raises(ValueError, match="max_nodes"):
            ss.ss_tree_mask([-1], n)
        with pytest.raises(ValueError, match="max_context"):
            ss.ss_attention_tree_workspace(4, 2, 64, 1, n, 1)
        with pytest.raises(ValueError, match="n_seq"):
            ss.ss_attention_tree_workspace(4, 2, 64, n, 100, 1)
        with pytest.raises(ValueError, match="max_len"):
            ss._count(n, "max_len")
    for slots in ([2**31], [3, 2**32 + 5], [-1], [[2, 3]]):
        with pytest.raises(ValueError, match="slots must be a list"):
            ss.Cache.allocate(slots, 1, 64, torch.int8, device="meta")
    for kv, dim in ((0, 64), (-2, 64), (2, 96)):
        with pytest.raises(ValueError, match="head_dim 64 or 128"):
            ss.Cache.allocate([4], kv, dim, torch.int8, device="meta")


def test_tables_of_trees_that_are_too_short_are_refused_by_the_binding(lib):
    """The library would read behind them.  (Without a model the whole ones are refused by the library, before it reads anything.)"""
    class NoModel:
        h, shape = None, type("Shape", (), dict(vocab=16))

    ok = dict(prompt_tokens=[1, 2, 3], prompt_offsets=[0, 2, 3], node_tokens=[4, 5], node_offsets=[0, 2, 2], parents=[-1, 0])
    for change in (dict(node_offsets=[0, 2]), dict(node_offsets=[0, 1, 2, 2]), dict(node_offsets=[]), dict(prompt_offsets=[0], node_offsets=[0]),
                   dict(prompt_offsets=[], node_offsets=[]), dict(prompt_tokens=[1, 2]), dict(node_tokens=[4]), dict(parents=[-1]), dict(node_offsets=[0, 2, -1])):
        with pytest.raises(ValueError, match="offsets"):
            ss.ss_tree_logits(NoModel, **{**ok, **change})
    with pytest.raises(ss.SsError) as e:
        ss.ss_tree_logits(NoModel, **ok)
    assert e.value.code == ss.SS_EINVAL

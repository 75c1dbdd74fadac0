"""The library's own calls on the cache operators: generation with keys and values held in 8 bits (SS_OPT_CACHE_BITS) and the logits
of drafted trees, against the oracle in 64 bits and against the calls that they must agree with.

The bar against the oracle is the library's own for teacher-forced logits, 3e-2 of the largest.  A code is off by at most half a
step, max|x| / 254: relative to a vector's norm about 2^-7 at most where its largest element is 4 times its mean one, and
independent between slots and elements, so that sums over them stay well inside."""
import numpy as np
import pytest

from oracle.model_oracle import OracleModel
from paper_2305_13144_amd import binding as ss
from paper_2305_13144_amd import synth

pytestmark = pytest.mark.gpu

SHAPES = {
    "tiny": synth.TINY,
    "wide": synth.ModelShape("wide", 2, 1024, 8, 128, 2048, 512),        # heads of 128; few rows, sweep and skinny kernels
}


@pytest.fixture(scope="module", params=sorted(SHAPES))
def model(request):
    shape = SHAPES[request.param]
    W = synth.make_weights(shape, seed=11, threads=4)
    gw = ss.Weights(shape, W)
    yield shape, gw, OracleModel(shape, W, "f64")
    gw.close()


def prompts(shape, lens, seed):
    rng = np.random.default_rng(seed)
    offs = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return rng.integers(0, shape.vocab, int(offs[-1])).astype(np.int32), offs


@pytest.mark.parametrize("lens,n_prompt", [([3], [1]), ([40, 2, 17, 90, 5], [30, 1, 17, 70, 4]), ([1100, 530, 20], [1094, 505, 14])])
def test_logits_with_an_8_bit_cache(model, lens, n_prompt):
    shape, gw, om = model
    toks, offs = prompts(shape, lens, len(lens))
    plain = ss.ss_forward_logits(gw, toks, offs, n_prompt)
    gw.set_option(ss.SS_OPT_CACHE_BITS, 8)
    try:
        got = ss.ss_forward_logits(gw, toks, offs, n_prompt)
        alone = ss.ss_forward_logits(gw, toks[:lens[0]], offs[:2], n_prompt[:1])
    finally:
        gw.set_option(ss.SS_OPT_CACHE_BITS, 16)
    ref = np.concatenate([om.teacher_forced(toks[offs[i]:offs[i + 1]], first=n_prompt[i] - 1) for i in range(len(lens))])
    assert np.abs(got - ref).max() <= 3e-2 * np.abs(ref).max()
    assert not np.array_equal(got, plain) or max(lens) < 4
    assert np.abs(alone - got[:len(alone)]).max() <= 2e-2 * np.abs(ref).max()       # other rows change launch shapes, no more
    again = ss.ss_forward_logits(gw, toks, offs, n_prompt)
    assert np.array_equal(again, plain)                                             # and the option leaves nothing behind


def test_many_rows_with_an_8_bit_cache(model):
    shape, gw, om = model
    lens = [int(n) for n in np.random.default_rng(5).integers(4, 40, 70)]
    n_prompt = [n - 3 for n in lens]
    toks, offs = prompts(shape, lens, 6)
    gw.set_option(ss.SS_OPT_CACHE_BITS, 8)
    try:
        got = ss.ss_forward_logits(gw, toks, offs, n_prompt)
    finally:
        gw.set_option(ss.SS_OPT_CACHE_BITS, 16)
    ref = np.concatenate([om.teacher_forced(toks[offs[i]:offs[i + 1]], first=n_prompt[i] - 1) for i in range(len(lens))])
    assert np.abs(got - ref).max() <= 3e-2 * np.abs(ref).max()


def test_one_head_and_odd_counts_of_slots_in_8_bits():
    """The codes of later layers lie behind the scales of earlier ones, here an odd number of 4-byte words."""
    shape = synth.ModelShape("one", 3, 64, 1, 64, 256, 256)
    W = synth.make_weights(shape, seed=3, threads=2)
    toks, offs = prompts(shape, [41, 12], 4)
    om = OracleModel(shape, W, "f64")
    gw = ss.Weights(shape, W)
    try:
        gw.set_option(ss.SS_OPT_CACHE_BITS, 8)
        got = ss.ss_forward_logits(gw, toks, offs, [30, 7])
    finally:
        gw.close()
    ref = np.concatenate([om.teacher_forced(toks[offs[i]:offs[i + 1]], first=n - 1) for i, n in enumerate((30, 7))])
    assert np.abs(got - ref).max() <= 3e-2 * np.abs(ref).max()


def test_generation_with_an_8_bit_cache(model):
    """Lengths, ends and counters are those of any cache; a row's tokens do not depend on flags, polling or the static workspace; and
    where the oracle's choice on the row's own prefix is clear, it is the row's."""
    shape, gw, om = model
    w = synth.make_group(shape, 12, 17, ("lognormal", 12.0, 0.6, 4, 60), ("lognormal", 12.0, 0.7, 1, 30), 0.3, 30, 8, (), base_batch=12, max_batch=16)
    gw.set_option(ss.SS_OPT_CACHE_BITS, 8)
    try:
        call = lambda flags=0, **kw: ss.ss_decode_microbatch(gw, w.prompt_tokens, w.prompt_offsets, 20, w.target_lens, flags, **kw)  # noqa: E731
        r = call()
        assert np.array_equal(r["lens"], np.minimum(w.target_lens, 20))
        assert np.array_equal(r["tokens"], call(ss.SS_COMPACT)["tokens"])
        s = call(static=True)
        assert np.array_equal(r["tokens"], s["tokens"]) and np.array_equal(r["failed"], s["failed"])
        g = ss.ss_generate_microbatch(gw, w.prompt_tokens, w.prompt_offsets, 20, target_lens=w.target_lens, sync_every=3, flags=ss.SS_COMPACT)
        assert np.array_equal(r["tokens"], g["tokens"]) and np.array_equal(r["lens"], g["lens"])
    finally:
        gw.set_option(ss.SS_OPT_CACHE_BITS, 16)
    clear = 0
    for i in range(w.n):
        L = int(r["lens"][i])
        seq = np.concatenate([w.prompt(i), r["tokens"][i, :L - 1]]).astype(np.int32)
        lg = om.teacher_forced(seq, first=len(w.prompt(i)) - 1)
        top = np.sort(lg, -1)
        sure = top[:, -1] - top[:, -2] > 6e-2 * np.abs(lg).max(-1)                   # twice the bar: both logits may be off
        assert (lg.argmax(-1)[sure] == r["tokens"][i, :L][sure]).all(), i
        clear += int(sure.sum())
    assert clear > 20


@pytest.mark.parametrize("flags", [(), ("SORT", "BIN", "FCR", "COMPACT")])
def test_a_group_with_an_8_bit_cache_does_not_depend_on_company(flags):
    shape = synth.LLAMA7B.with_layers(1)
    gw = ss.Weights(shape, synth.make_weights(shape, seed=3, threads=8))
    w = synth.make_group(shape, 60, 92, ("lognormal", 30.0, 0.6, 4, 600), ("lognormal", 12.0, 0.7, 1, 40), 0.3, 40, 8, flags, base_batch=16, max_batch=48)
    pol = ss.make_policy(flags, 16, 40, 48)
    preds = w.pred_lens if flags else None
    gw.set_option(ss.SS_OPT_CACHE_BITS, 8)
    got = []
    for lanes in (1, 4):
        gw.set_option(ss.SS_OPT_IN_FLIGHT, lanes)
        got.append(ss.ss_run_group(gw, w.prompt_tokens, w.prompt_offsets, w.target_lens, preds, 8 if flags else 0, pol))
        assert np.array_equal(got[-1]["lens"], w.target_lens)
    assert np.array_equal(got[0]["tokens"], got[1]["tokens"])
    ms = ss.ss_bench_decode_step(gw, np.zeros(2 * 600, np.int32), 2, 600, 2)
    assert (ms > 0).all()
    gw.close()


def test_the_other_entry_points_with_an_8_bit_cache(model):
    """Sampled groups do not depend on lanes, logits of prompts are near the oracle's, and the measurements run."""
    shape, gw, om = model
    w = synth.make_group(shape, 20, 31, ("uniform", 4, 40), ("lognormal", 8.0, 0.6, 1, 20), 0.3, 20, 8, ("SORT", "BIN"), base_batch=8, max_batch=16)
    toks, offs = prompts(shape, [25, 3], 9)
    gw.set_option(ss.SS_OPT_CACHE_BITS, 8)
    try:
        got = []
        for lanes in (1, 3):
            gw.set_option(ss.SS_OPT_IN_FLIGHT, lanes)
            got.append(ss.ss_run_group_generate(gw, w.prompt_tokens, w.prompt_offsets, w.pred_lens, 8, ss.make_policy(("SORT", "BIN"), 8, 20, 16),
                                                temperature=0.7, seed=5, target_lens=w.target_lens))
        everything = ss.ss_forward_logits(gw, toks, offs, [25, 3], all_prompt_logits=True)
        assert (ss.ss_bench_decode_steps_in_flight(gw, np.zeros(3 * 50, np.int32), 3, 50, 2) > 0).all()
        assert (ss.ss_bench_weight_stream(gw, 3, 2)[0] > 0).all()
    finally:
        gw.set_option(ss.SS_OPT_CACHE_BITS, 16)
        gw.set_option(ss.SS_OPT_IN_FLIGHT, 4)
    assert np.array_equal(got[0]["tokens"], got[1]["tokens"]) and np.array_equal(got[0]["lens"], got[1]["lens"])
    ref = np.concatenate([om.teacher_forced(toks[offs[i]:offs[i + 1]], first=0) for i in range(2)])
    assert everything.shape == ref.shape and np.abs(everything - ref).max() <= 3e-2 * np.abs(ref).max()


def test_the_option_takes_8_and_16(model):
    shape, gw, om = model
    for bad in (0, 1, 4, 32, -8):
        with pytest.raises(ss.SsError) as e:
            gw.set_option(ss.SS_OPT_CACHE_BITS, bad)
        assert e.value.code == ss.SS_EINVAL


# ------------------------------------------------------------------------------------------------ drafted trees
def random_tree(rng, n):
    return [int(rng.integers(-1, t)) if t else -1 for t in range(n)]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("lens,nodes", [([5], [1]), ([7, 30, 1, 12], [9, 0, 33, 1]), ([600, 3], [20, 70]), ([4, 6], [0, 0])])
def test_logits_of_trees(model, bits, lens, nodes):
    """Every node's logits are those that its path through the tree has as an ordinary sequence."""
    shape, gw, om = model
    rng = np.random.default_rng(sum(lens) + sum(nodes))
    toks, offs = prompts(shape, lens, 3)
    noffs = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    parents = np.array([p for n in nodes for p in random_tree(rng, n)], np.int32)
    ntoks = rng.integers(0, shape.vocab, int(noffs[-1])).astype(np.int32)
    gw.set_option(ss.SS_OPT_CACHE_BITS, bits)
    try:
        got = ss.ss_tree_logits(gw, toks, offs, ntoks, noffs, parents)
        again = ss.ss_tree_logits(gw, toks, offs, ntoks, noffs, parents)
    finally:
        gw.set_option(ss.SS_OPT_CACHE_BITS, 16)
    assert np.array_equal(got, again)
    at = 0
    for i in range(len(lens)):
        prompt = toks[offs[i]:offs[i + 1]]
        ref = om.teacher_forced(prompt, first=lens[i] - 1)
        assert np.abs(got[at] - ref[0]).max() <= 3e-2 * np.abs(ref).max()
        for t in range(nodes[i]):
            path, u = [], t
            while u >= 0:
                path.append(ntoks[noffs[i] + u])
                u = int(parents[noffs[i] + u])
            ref = om.teacher_forced(np.concatenate([prompt, path[::-1]]).astype(np.int32), first=lens[i] + len(path) - 1)
            assert np.abs(got[at + 1 + t] - ref[0]).max() <= 3e-2 * np.abs(ref).max(), (i, t)
        at += 1 + nodes[i]


def test_a_chain_has_the_logits_of_its_tokens_one_by_one(model):
    shape, gw, om = model
    toks, offs = prompts(shape, [20, 33], 8)
    chain = [4, 7]
    at = [(0, 16, 20), (20, 46, 53)]                              # prompt, drafted part of the same sequences
    ptoks = np.concatenate([toks[a:b] for a, b, _ in at])
    ntoks = np.concatenate([toks[b:c] for _, b, c in at])
    got = ss.ss_tree_logits(gw, ptoks, [0, 16, 42], ntoks, [0, 4, 11], [-1, 0, 1, 2, -1, 0, 1, 2, 3, 4, 5])
    ref = ss.ss_forward_logits(gw, toks, offs, [16, 26])
    assert got.shape == ref.shape and sum(chain) + 2 == len(ref)
    assert np.abs(got - ref).max() <= 1e-2 * np.abs(ref).max()    # other launch shapes (1e-3 each way), queries rounded to half


def test_bad_trees_are_refused(model):
    shape, gw, om = model
    ok = dict(prompt_tokens=[1, 2, 3], prompt_offsets=[0, 3], node_tokens=[4, 5], node_offsets=[0, 2], parents=[-1, 0])
    assert ss.ss_tree_logits(gw, **ok).shape == (3, shape.vocab)
    for change in (dict(parents=[-1, 1]), dict(parents=[0, 0]), dict(parents=[-2, 0]), dict(node_tokens=[4, shape.vocab]), dict(node_tokens=[-1, 5]),
                   dict(node_offsets=[1, 2]), dict(prompt_offsets=[0, 0]), dict(prompt_tokens=[1, 2, -3]),
                   dict(prompt_tokens=[1] * 4095, prompt_offsets=[0, 4095])):
        with pytest.raises(ss.SsError) as e:
            ss.ss_tree_logits(gw, **{**ok, **change})
        assert e.value.code == ss.SS_EINVAL, change
    with pytest.raises(ss.SsError):
        ss.ss_tree_logits(gw, [1], [0, 1], [1] * 1025, [0, 1025], [-1] * 1025)
    assert ss.ss_tree_logits(gw, **ok).shape == (3, shape.vocab)

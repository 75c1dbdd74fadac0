"""ctypes binding of libss.so: argument marshalling only, same names as the C ABI.

Every step of the path runs in the library's kernels; nothing here computes.  The library
must be built (``python -m paper_2305_13144_amd.build``) - there is no fallback: a missing
library raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import NamedTuple, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libss.so")

SS_OK, SS_EINVAL, SS_ENOMEM, SS_EDEVICE, SS_ESTATE = 0, -1, -2, -3, -4
SS_SORT, SS_BIN, SS_FCR, SS_VBS, SS_COMPACT = 1, 2, 4, 8, 16
SS_VBS_CLAMP_FLOOR, SS_VBS_PAPER_POW2 = 0, 1
SS_OPT_IN_FLIGHT, SS_IN_FLIGHT_MAX, SS_IN_FLIGHT_DEFAULT = 2, 4, 4
SS_OPT_WEIGHT_COPIES, SS_OPT_CACHE_BITS = 3, 4
SS_BF16, SS_F32, SS_F16, SS_I8 = 0, 1, 2, 3
SS_TREE_MAX_NODES = 1024
SS_PAGES_MAX, SS_PAGES_MAX_ROWS, SS_PAGES_MAX_GROUP, SS_BEAM_MAX = 1 << 27, 8192, 32, 64
FLAG_BITS = dict(SORT=SS_SORT, BIN=SS_BIN, FCR=SS_FCR, VBS=SS_VBS, COMPACT=SS_COMPACT)

EXPORTS = ["ss_last_error", "ss_set_verbose", "ss_set_gemm_mode", "ss_schedule", "ss_schedule_failures", "ss_plan_free", "ss_weights_create",
           "ss_weights_destroy", "ss_set_option", "ss_decode_microbatch", "ss_decode_microbatch_static", "ss_forward_logits", "ss_tree_logits", "ss_run_group", "ss_generate_microbatch",
           "ss_run_group_generate", "ss_bench_decode_step", "ss_bench_decode_steps_in_flight", "ss_bench_weight_stream", "ss_bench_read_stream",
           "ss_cache_write", "ss_cache_read", "ss_attention_tree", "ss_attention_tree_workspace", "ss_tree_mask", "ss_attention_packed",
           "ss_pages_write", "ss_pages_read", "ss_attention_pages", "ss_attention_pages_workspace", "ss_pages_fork", "ss_pages_compact",
           "ss_pages_workspace", "ss_pages_copy", "ss_beam_select", "ss_beam_select_workspace"]


class SsError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libss error {code}: {msg}")
        self.code = code


class ss_policy(C.Structure):
    _fields_ = [("flags", C.c_uint32), ("base_batch", C.c_int32), ("base_len", C.c_int32), ("max_batch", C.c_int32),
                ("vbs_rule", C.c_int32)]


class ss_plan(C.Structure):
    _fields_ = [("n", C.c_int32), ("n_mb", C.c_int32), ("mb_offsets", C.POINTER(C.c_int32)),
                ("query_idx", C.POINTER(C.c_int32)), ("mb_cap", C.POINTER(C.c_int32))]


class ss_model_cfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
                ("d_ffn", C.c_int32), ("vocab", C.c_int32), ("rope_base", C.c_float), ("rms_eps", C.c_float)]


class ss_stats(C.Structure):
    _fields_ = [("steps", C.c_int32), ("rows", C.c_int32), ("row_steps", C.c_int64), ("prompt_tokens", C.c_int64),
                ("decode_kv_tokens", C.c_int64), ("prefill_ms", C.c_double), ("decode_ms", C.c_double),
                ("polls", C.c_int32), ("idle_steps", C.c_int32)]


class ss_group_stats(C.Structure):
    _fields_ = [("n_mb_first", C.c_int32), ("n_mb_failure", C.c_int32), ("n_failed", C.c_int32),
                ("steps", C.c_int64), ("padded_row_steps", C.c_int64), ("computed_row_steps", C.c_int64),
                ("useful_tokens", C.c_int64), ("prompt_tokens", C.c_int64), ("wall_ms", C.c_double),
                ("plan_ms", C.c_double), ("prefill_ms", C.c_double), ("decode_ms", C.c_double),
                ("polls", C.c_int64), ("idle_steps", C.c_int64)]


class ss_gen_opts(C.Structure):
    _fields_ = [("eos_id", C.c_int32), ("temperature", C.c_float), ("draws", C.c_void_p),
                ("draws_stride", C.c_int32), ("seed", C.c_uint64), ("draw_ids", C.c_void_p),
                ("target_lens", C.c_void_p), ("sync_every", C.c_int32)]


class ss_rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64), ("rows", C.c_int64), ("dtype", C.c_int32)]


class ss_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("start", C.c_void_p),
                ("slots", C.c_void_p), ("total_slots", C.c_int64), ("n_seq", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class ss_pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("n_pages", C.c_int32),
                ("page_slots", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class ss_page_table(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("lengths", C.c_void_p), ("n_rows", C.c_int32), ("stride", C.c_int32),
                ("page_slots", C.c_int32), ("n_pages", C.c_int32)]


class ss_beams(C.Structure):
    _fields_ = [("totals", C.c_void_p), ("lengths", C.c_void_p), ("ended", C.c_void_p), ("history", C.c_void_p),
                ("history_stride", C.c_int32)]


def _struct_dict(s: C.Structure) -> dict:
    return {name: getattr(s, name) for name, _ in s._fields_}


_lib = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: build it with `python -m paper_2305_13144_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32p = C.c_void_p, C.c_void_p
        L.ss_last_error.restype = C.c_char_p
        L.ss_set_verbose.argtypes = [C.c_int32]
        L.ss_set_verbose.restype = None
        L.ss_set_gemm_mode.argtypes = [C.c_int32]
        L.ss_set_gemm_mode.restype = None
        L.ss_schedule.argtypes = [i32p, C.c_int32, C.c_int32, C.POINTER(ss_policy), C.POINTER(C.POINTER(ss_plan))]
        L.ss_schedule_failures.argtypes = [i32p, C.c_int32, i32p, C.c_int32, C.c_int32, C.POINTER(ss_policy),
                                           C.POINTER(C.POINTER(ss_plan))]
        L.ss_plan_free.argtypes = [C.POINTER(ss_plan)]
        L.ss_plan_free.restype = None
        L.ss_weights_create.argtypes = [C.POINTER(ss_model_cfg), C.POINTER(vp), C.c_int32, C.POINTER(vp)]
        L.ss_set_option.argtypes = [vp, C.c_int32, C.c_int32]
        L.ss_weights_destroy.argtypes = [vp]
        L.ss_weights_destroy.restype = None
        L.ss_decode_microbatch.argtypes = [vp, i32p, i32p, C.c_int32, C.c_int32, i32p, C.c_uint32, i32p, i32p, vp,
                                           C.POINTER(ss_stats), vp]
        L.ss_decode_microbatch_static.argtypes = L.ss_decode_microbatch.argtypes
        L.ss_forward_logits.argtypes = [vp, i32p, i32p, C.c_int32, i32p, C.c_int32, vp, vp]
        L.ss_tree_logits.argtypes = [vp, i32p, i32p, C.c_int32, i32p, i32p, i32p, vp, vp]
        L.ss_run_group.argtypes = [vp, i32p, i32p, C.c_int32, i32p, i32p, C.c_int32, C.POINTER(ss_policy), i32p, i32p,
                                   C.POINTER(ss_group_stats), vp]
        L.ss_generate_microbatch.argtypes = [vp, i32p, i32p, C.c_int32, C.c_int32, C.POINTER(ss_gen_opts), C.c_uint32,
                                             i32p, i32p, vp, C.POINTER(ss_stats), vp]
        L.ss_run_group_generate.argtypes = [vp, i32p, i32p, C.c_int32, i32p, C.c_int32, C.POINTER(ss_policy),
                                            C.POINTER(ss_gen_opts), i32p, i32p, C.POINTER(ss_group_stats), vp]
        L.ss_bench_decode_step.argtypes = [vp, i32p, C.c_int32, C.c_int32, C.c_int32, vp, vp]
        L.ss_bench_decode_steps_in_flight.argtypes = [vp, i32p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, vp]
        L.ss_bench_weight_stream.argtypes = [vp, C.c_int32, C.c_int32, vp, vp, vp]
        L.ss_bench_read_stream.argtypes = [vp, C.c_int32, vp, vp, vp]
        rows, cache = C.POINTER(ss_rows), C.POINTER(ss_cache)
        L.ss_cache_write.argtypes = [cache, rows, rows, vp, vp, C.c_int32, vp]
        L.ss_cache_read.argtypes = [cache, vp, vp, C.c_int32, rows, rows, vp]
        L.ss_attention_tree.argtypes = [cache, rows, rows, C.c_int32, C.c_int32, vp, vp, C.c_int32, vp, C.c_int32, vp, C.c_float,
                                        vp, C.c_size_t, vp]
        L.ss_attention_tree_workspace.argtypes = [C.c_int32] * 6 + [C.POINTER(C.c_size_t)]
        L.ss_tree_mask.argtypes = [vp, C.c_int32, C.c_int32, vp]
        L.ss_attention_packed.argtypes = [rows, rows, rows, rows, C.c_int32, C.c_int32, C.c_int32, vp, C.c_int32, C.c_int32,
                                          C.c_float, vp]
        pages, table, beams, i32 = C.POINTER(ss_pages), C.POINTER(ss_page_table), C.POINTER(ss_beams), C.c_int32
        L.ss_pages_write.argtypes = [pages, table, rows, rows, vp, vp, i32, vp]
        L.ss_pages_read.argtypes = [pages, table, vp, vp, i32, rows, rows, vp]
        L.ss_attention_pages.argtypes = [pages, table, rows, rows, i32, i32, vp, i32, i32, C.c_float, vp, C.c_size_t, vp]
        L.ss_attention_pages_workspace.argtypes = [i32] * 8 + [C.POINTER(C.c_size_t)]
        L.ss_pages_fork.argtypes = [table, table, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.ss_pages_compact.argtypes = [table, table, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.ss_pages_workspace.argtypes = [i32, C.POINTER(C.c_size_t)]
        L.ss_pages_copy.argtypes = [pages, i32, vp, vp, i32, vp, vp]
        L.ss_beam_select.argtypes = [vp, i32, C.c_int64, i32, i32, i32, i32, beams, beams, vp, vp, i32, C.c_float, vp, C.c_size_t, vp]
        L.ss_beam_select_workspace.argtypes = [i32] * 4 + [C.POINTER(C.c_size_t)]
        for name in EXPORTS:
            if name not in ("ss_last_error", "ss_set_verbose", "ss_set_gemm_mode", "ss_plan_free", "ss_weights_destroy"):
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _check(rc: int) -> None:
    if rc != SS_OK:
        raise SsError(rc, lib().ss_last_error().decode())


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int32)


def _ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def ss_set_verbose(level: int) -> None:
    lib().ss_set_verbose(level)


def ss_set_gemm_mode(mode: int) -> None:
    lib().ss_set_gemm_mode(mode)


def make_policy(flags: Sequence[str] = (), base_batch: int = 16, base_len: int = 512, max_batch: int = 256,
                vbs_rule: int = SS_VBS_CLAMP_FLOOR) -> ss_policy:
    bits = 0
    for f in flags:
        bits |= FLAG_BITS[f]
    return ss_policy(bits, base_batch, base_len, max_batch, vbs_rule)


def _plan_to_py(pp) -> list:
    p = pp.contents
    offs = [p.mb_offsets[i] for i in range(p.n_mb + 1)]
    idx = [p.query_idx[i] for i in range(p.n)]
    out = [(idx[offs[k]:offs[k + 1]], p.mb_cap[k]) for k in range(p.n_mb)]
    lib().ss_plan_free(pp)
    return out


def ss_schedule(pred_lens, n: int, bin: int, policy: ss_policy) -> list:
    """-> [(query indices, cap), ...] in execution order."""
    pl = None if pred_lens is None else _i32(pred_lens)
    out = C.POINTER(ss_plan)()
    _check(lib().ss_schedule(_ptr(pl), n, bin, C.byref(policy), C.byref(out)))
    return _plan_to_py(out)


def ss_schedule_failures(pred_lens, n: int, failed_idx, bin: int, policy: ss_policy) -> list:
    pl = None if pred_lens is None else _i32(pred_lens)
    fi = _i32(failed_idx)
    out = C.POINTER(ss_plan)()
    _check(lib().ss_schedule_failures(_ptr(pl), n, _ptr(fi), len(fi), bin, C.byref(policy), C.byref(out)))
    return _plan_to_py(out)


class Weights:
    """Owns an ss_weights handle (device-resident packed model)."""

    def __init__(self, shape, tensors: Sequence[np.ndarray], src_dtype: int = SS_BF16):
        want = np.uint16 if src_dtype == SS_BF16 else np.float32
        self._keep = [np.ascontiguousarray(t, dtype=want) for t in tensors]
        n_expected = 3 + 9 * shape.n_layers
        if len(self._keep) != n_expected:
            raise ValueError(f"expected {n_expected} tensors, got {len(self._keep)}")
        cfg = ss_model_cfg(shape.n_layers, shape.d_model, shape.n_heads, shape.head_dim, shape.d_ffn, shape.vocab,
                           shape.rope_base, shape.rms_eps)
        arr = (C.c_void_p * len(self._keep))(*[t.ctypes.data for t in self._keep])
        h = C.c_void_p()
        _check(lib().ss_weights_create(C.byref(cfg), arr, src_dtype, C.byref(h)))
        self.h = h
        self.shape = shape
        self._keep = None   # the library copied everything

    def set_option(self, option: int, value: int) -> None:
        _check(lib().ss_set_option(self.h, option, value))

    def close(self) -> None:
        if getattr(self, "h", None):
            lib().ss_weights_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def ss_decode_microbatch(w: Weights, prompt_tokens, prompt_offsets, max_new: int, target_lens, flags: int = 0,
                         stream: Optional[int] = None, static: bool = False) -> dict:
    """static=True calls ss_decode_microbatch_static (workspace in the library's static device array)."""
    pt, po, tl = _i32(prompt_tokens), _i32(prompt_offsets), _i32(target_lens)
    B = len(tl)
    toks = np.empty((B, max_new), np.int32)
    lens = np.empty(B, np.int32)
    failed = np.empty(B, np.uint8)
    st = ss_stats()
    fn = lib().ss_decode_microbatch_static if static else lib().ss_decode_microbatch
    _check(fn(w.h, _ptr(pt), _ptr(po), B, max_new, _ptr(tl), flags, _ptr(toks), _ptr(lens), _ptr(failed), C.byref(st),
              stream))
    return dict(tokens=toks, lens=lens, failed=failed, stats=_struct_dict(st))


def ss_decode_microbatch_static(w: Weights, prompt_tokens, prompt_offsets, max_new: int, target_lens, flags: int = 0,
                                stream: Optional[int] = None) -> dict:
    return ss_decode_microbatch(w, prompt_tokens, prompt_offsets, max_new, target_lens, flags, stream, static=True)


def ss_forward_logits(w: Weights, tokens, offsets, n_prompt, all_prompt_logits: bool = False,
                      stream: Optional[int] = None) -> np.ndarray:
    tk, of, npz = _i32(tokens), _i32(offsets), _i32(n_prompt)
    B = len(npz)
    lens = np.diff(of)
    rows = int(lens.sum()) if all_prompt_logits else int((lens - npz + 1).sum())
    out = np.empty((rows, w.shape.vocab), np.float32)
    _check(lib().ss_forward_logits(w.h, _ptr(tk), _ptr(of), B, _ptr(npz), int(all_prompt_logits), _ptr(out), stream))
    return out


def ss_tree_logits(w: Weights, prompt_tokens, prompt_offsets, node_tokens, node_offsets, parents, stream: Optional[int] = None) -> np.ndarray:
    """[B + nodes, vocab]: for each row the logits of its prompt's last position, then those of its drafted nodes."""
    pt, po, nt, no, pa = (_i32(a) for a in (prompt_tokens, prompt_offsets, node_tokens, node_offsets, parents))
    B = len(po) - 1
    if B < 1 or len(no) != B + 1:
        raise ValueError(f"prompt_offsets and node_offsets must both have rows + 1 entries: they have {len(po)} and {len(no)}")
    if len(pt) < po[-1] or no[-1] < 0 or len(nt) < no[-1] or len(pa) < no[-1]:
        raise ValueError(f"{len(pt)} prompt tokens, {len(nt)} node tokens and {len(pa)} parents are fewer than the offsets say ({po[-1]}, {no[-1]}, {no[-1]})")
    out = np.empty((B + int(no[-1]), w.shape.vocab), np.float32)
    _check(lib().ss_tree_logits(w.h, _ptr(pt), _ptr(po), B, _ptr(nt), _ptr(no), _ptr(pa), _ptr(out), stream))
    return out


def ss_run_group(w: Weights, prompt_tokens, prompt_offsets, target_lens, pred_lens, bin: int, policy: ss_policy,
                 stream: Optional[int] = None) -> dict:
    pt, po, tl = _i32(prompt_tokens), _i32(prompt_offsets), _i32(target_lens)
    pl = None if pred_lens is None else _i32(pred_lens)
    n = len(tl)
    toks = np.empty((n, policy.base_len), np.int32)
    lens = np.zeros(n, np.int32)
    gs = ss_group_stats()
    _check(lib().ss_run_group(w.h, _ptr(pt), _ptr(po), n, _ptr(tl), _ptr(pl), bin, C.byref(policy), _ptr(toks),
                              _ptr(lens), C.byref(gs), stream))
    return dict(tokens=toks, lens=lens, stats=_struct_dict(gs))


def _gen_opts(eos_id: int, temperature: float, draws, target_lens, sync_every: int, seed: int = 0, draw_ids=None):
    """Marshals ss_gen_opts; returns (struct, arrays to keep alive)."""
    d = None if draws is None else np.ascontiguousarray(draws, dtype=np.float32)
    tl = None if target_lens is None else _i32(target_lens)
    ids = None if draw_ids is None else _i32(draw_ids)
    o = ss_gen_opts()
    o.seed = int(seed)
    o.draw_ids = None if ids is None else ids.ctypes.data
    o.eos_id, o.temperature, o.sync_every = int(eos_id), float(temperature), int(sync_every)
    o.draws = None if d is None else d.ctypes.data
    o.draws_stride = 0 if d is None else int(d.shape[1])
    o.target_lens = None if tl is None else tl.ctypes.data
    return o, (d, tl, ids)


def ss_generate_microbatch(w: Weights, prompt_tokens, prompt_offsets, max_new: int, eos_id: int = -1,
                           temperature: float = 0.0, draws=None, target_lens=None, sync_every: int = 8,
                           flags: int = 0, seed: int = 0, draw_ids=None, stream: Optional[int] = None) -> dict:
    pt, po = _i32(prompt_tokens), _i32(prompt_offsets)
    B = len(po) - 1
    opts, keep = _gen_opts(eos_id, temperature, draws, target_lens, sync_every, seed, draw_ids)
    toks = np.empty((B, max_new), np.int32)
    lens = np.empty(B, np.int32)
    failed = np.empty(B, np.uint8)
    st = ss_stats()
    _check(lib().ss_generate_microbatch(w.h, _ptr(pt), _ptr(po), B, max_new, C.byref(opts), flags, _ptr(toks),
                                        _ptr(lens), _ptr(failed), C.byref(st), stream))
    del keep
    return dict(tokens=toks, lens=lens, failed=failed, stats=_struct_dict(st))


def ss_run_group_generate(w: Weights, prompt_tokens, prompt_offsets, pred_lens, bin: int, policy: ss_policy,
                          eos_id: int = -1, temperature: float = 0.0, draws=None, target_lens=None,
                          sync_every: int = 8, seed: int = 0, draw_ids=None, stream: Optional[int] = None) -> dict:
    pt, po = _i32(prompt_tokens), _i32(prompt_offsets)
    pl = None if pred_lens is None else _i32(pred_lens)
    n = len(po) - 1
    opts, keep = _gen_opts(eos_id, temperature, draws, target_lens, sync_every, seed, draw_ids)
    toks = np.empty((n, policy.base_len), np.int32)
    lens = np.zeros(n, np.int32)
    gs = ss_group_stats()
    _check(lib().ss_run_group_generate(w.h, _ptr(pt), _ptr(po), n, _ptr(pl), bin, C.byref(policy), C.byref(opts),
                                       _ptr(toks), _ptr(lens), C.byref(gs), stream))
    del keep
    return dict(tokens=toks, lens=lens, stats=_struct_dict(gs))


def ss_bench_decode_step(w: Weights, prompt_tokens, B: int, ctx: int, iters: int,
                         stream: Optional[int] = None) -> np.ndarray:
    pt = _i32(prompt_tokens)
    assert pt.size == B * ctx
    ms = np.empty(iters, np.float64)
    _check(lib().ss_bench_decode_step(w.h, _ptr(pt), B, ctx, iters, _ptr(ms), stream))
    return ms


def ss_bench_decode_steps_in_flight(w: Weights, prompt_tokens, B: int, ctx: int, iters: int, lanes: int = 2) -> np.ndarray:
    """[lanes, iters] device milliseconds: the lanes' decode forwards running at the same time."""
    pt = _i32(prompt_tokens)
    assert pt.size == B * ctx
    ms = np.zeros(lanes * iters, np.float64)
    _check(lib().ss_bench_decode_steps_in_flight(w.h, _ptr(pt), B, ctx, iters, lanes, _ptr(ms)))
    return ms.reshape(lanes, iters)


def ss_bench_weight_stream(w: Weights, B: int, iters: int, stream: Optional[int] = None):
    ms = np.empty(iters, np.float64)
    launches = C.c_int32(0)
    _check(lib().ss_bench_weight_stream(w.h, B, iters, _ptr(ms), C.byref(launches), stream))
    return ms, int(launches.value)


def ss_bench_read_stream(w: Weights, iters: int, stream: Optional[int] = None):
    ms = np.empty(iters, np.float64)
    nbytes = C.c_int64(0)
    _check(lib().ss_bench_read_stream(w.h, iters, _ptr(ms), C.byref(nbytes), stream))
    return ms, int(nbytes.value)


# ---------------------------------------------------------------------------------------------------- operators on device tensors
# Tensors are torch's, used where they lie: nothing is copied.  The calls go to torch's current stream of the tensors' device and return once
# enqueued.  Given another `stream` (a HIP stream handle, 0: the default stream) they go there, behind what the current stream holds so
# far, and the tensors' memory is not given to others before that work is done; whoever reads the results on another
# stream has it wait for this one, as with torch's own.  (A graph that is being captured there cannot wait for work outside it.)
# Forward only: tensors that require gradients are refused unless gradients are off (torch.no_grad(), or detach()).

_torch = None
_raw_stream = None
_ELEMENT = {}   # torch dtype -> element type


def _with_torch():
    """torch, with the library on the same HIP runtime: pointers and streams of another one mean nothing to it."""
    global _torch, _raw_stream
    if _torch is None:
        import torch

        lib()
        with open("/proc/self/maps") as f:
            runtimes = {line.split()[-1] for line in f if "libamdhip64" in line}
        if len(runtimes) > 1:
            raise RuntimeError("torch and this library have loaded a HIP runtime each (" + ", ".join(sorted(runtimes)) +
                               "): import torch before the library is first used")
        _ELEMENT.update({torch.float16: SS_F16, torch.bfloat16: SS_BF16, torch.int8: SS_I8})
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # a microsecond less than current_stream()
        _torch = torch
    return _torch


def _refuse(t, name: str, index: int, what: str):
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU: it is on {t.device}")
    if t.get_device() != index:
        raise ValueError(f"{name} must be on cuda:{index}: it is on {t.device}")
    raise ValueError(f"{name} must be {what}: it is {list(t.shape)} of {t.dtype} with strides {list(t.stride())}")


def _rows(t, name: str, index: int, heads: Optional[int], head_dim: int) -> ss_rows:
    """[rows, heads, head_dim] of float16 or bfloat16 with any strides but the last; on device `index`."""
    if t.requires_grad and _torch.is_grad_enabled():
        raise ValueError(f"{name} requires gradients, and this operator has none: call it under torch.no_grad(), or with {name}.detach()")
    shape, dtype = t.shape, _ELEMENT.get(t.dtype, SS_I8)
    if t.get_device() != index or len(shape) != 3 or shape[2] != head_dim or (heads is not None and shape[1] != heads) or dtype == SS_I8:
        _refuse(t, name, index, f"[rows, {'heads' if heads is None else heads}, {head_dim}] of float16 or bfloat16")
    r, h, e = t.stride()
    if e != 1:
        _refuse(t, name, index, "a tensor whose last dimension is contiguous")
    return ss_rows(t.data_ptr(), r, h, shape[0], dtype)


def _table(t, name: str, index: int, count: int, dtype):
    if t is None:
        return None
    if t.get_device() != index or t.dtype is not dtype or t.numel() != count or not t.is_contiguous():
        _refuse(t, name, index, f"{count} contiguous values of {dtype}")
    return t.data_ptr()


def _stream(index: int) -> int:
    """Handle of torch's current stream."""
    return _raw_stream(index) if _raw_stream else _torch.cuda.current_stream(index).cuda_stream


def _on(stream: Optional[int], index: int, *tensors) -> int:
    """Handle of the stream that a call goes to, given one or none, in order behind the current one and with the tensors kept."""
    now = _stream(index)
    if stream is None or stream == now:
        return now
    t = _torch.cuda
    there = t.ExternalStream(stream, device=index) if stream else t.default_stream(index)
    with t.stream(there):
        captured = t.is_current_stream_capturing()
    if not captured or t.is_current_stream_capturing():
        there.wait_stream(t.current_stream(index))
    for x in tensors:
        if x is not None:
            x.record_stream(there)
    return stream


def _count(n: int, name: str) -> int:
    """An argument of 32 bits: ctypes would cut a larger one to another number."""
    if not -2**31 <= n < 2**31:
        raise ValueError(f"{name} must be a number of 32 bits: it is {n}")
    return n


class Cache:
    """The key/value cache of one layer (ss_cache): a view of tensors that the caller owns.

    k, v              flat, total slots * n_kv_heads * head_dim elements of float16, bfloat16 or int8
    start, slots      int64 and int32 [sequences]: first slot and number of slots of each sequence's slab
    k_scale, v_scale  flat float32, total slots * n_kv_heads, with int8
    """

    def __init__(self, k, v, start, slots, n_kv_heads: int, head_dim: int, k_scale=None, v_scale=None):
        t = _with_torch()
        if n_kv_heads < 1 or head_dim not in (64, 128):
            raise ValueError("n_kv_heads must be positive, head_dim 64 or 128")
        if k.dtype not in _ELEMENT or not k.is_cuda or k.numel() % (n_kv_heads * head_dim):
            _refuse(k, "k", k.get_device(), "whole slots of float16, bfloat16 or int8")
        index, n, dtype = k.get_device(), start.numel(), _ELEMENT[k.dtype]
        total = k.numel() // (n_kv_heads * head_dim)
        if (dtype == SS_I8) != (k_scale is not None) or (dtype == SS_I8) != (v_scale is not None):
            raise ValueError("k_scale and v_scale belong to int8 caches, and only to them")
        ptr = [_table(x, name, index, k.numel(), k.dtype) for x, name in ((k, "k"), (v, "v"))]
        ptr += [_table(x, name, index, total * n_kv_heads, t.float32) for x, name in ((k_scale, "k_scale"), (v_scale, "v_scale"))]
        ptr += [_table(start, "start", index, n, t.int64), _table(slots, "slots", index, n, t.int32)]
        self.k, self.v, self.k_scale, self.v_scale, self.start, self.slots = k, v, k_scale, v_scale, start, slots
        self.n_seq, self.n_kv_heads, self.head_dim, self.total_slots = n, n_kv_heads, head_dim, total
        self.device, self.index = k.device, index
        self.struct = ss_cache(*ptr, total, n, n_kv_heads, head_dim, dtype)
        self.tensors = (k, v, start, slots, k_scale, v_scale)

    @classmethod
    def allocate(cls, slots: Sequence[int], n_kv_heads: int, head_dim: int, dtype, device="cuda") -> "Cache":
        """An empty cache of torch.float16, bfloat16 or int8 with a slab of slots[i] slots for sequence i, one behind the other."""
        t = _with_torch()
        n = np.asarray(slots, dtype=np.int64)
        if n.ndim != 1 or (n < 0).any() or (n >= 2**31).any():
            raise ValueError("slots must be a list of numbers >= 0 and below 2^31")
        if n_kv_heads < 1 or head_dim not in (64, 128):
            raise ValueError("n_kv_heads must be positive, head_dim 64 or 128")
        total = int(n.sum())
        k, v = (t.zeros(total * n_kv_heads * head_dim, dtype=dtype, device=device) for _ in range(2))
        scales = [t.zeros(total * n_kv_heads, device=device) if dtype == t.int8 else None for _ in range(2)]
        start = t.from_numpy(np.cumsum(n) - n).to(device)
        return cls(k, v, start, t.from_numpy(n.astype(np.int32)).to(device), n_kv_heads, head_dim, *scales)


def ss_cache_write(cache: Cache, k, v, seq, slot, stream: Optional[int] = None) -> None:
    """Keys and values [n, n_kv_heads, head_dim] of n tokens to slot[t] of sequence seq[t] (int32 [n]; -1: passed over)."""
    t, index = _torch, cache.index
    if index != t.cuda.current_device():
        with t.cuda.device(index):
            return ss_cache_write(cache, k, v, seq, slot, stream)
    n, kv, hd, i32 = k.shape[0], cache.n_kv_heads, cache.head_dim, t.int32
    _check(_lib.ss_cache_write(cache.struct, _rows(k, "k", index, kv, hd), _rows(v, "v", index, kv, hd), _table(seq, "seq", index, n, i32),
                               _table(slot, "slot", index, n, i32), n, _on(stream, index, k, v, seq, slot, *cache.tensors)))


def ss_cache_read(cache: Cache, seq, slot, dtype=None, k=None, v=None, stream: Optional[int] = None):
    """(k, v) [n, n_kv_heads, head_dim]: what slot[t] of sequence seq[t] stands for.  Into k and v if they are given, whose rows of
    tokens that do not exist stay as they are; into new tensors of `dtype` (float16) otherwise, where those rows are undefined."""
    t, index = _torch, cache.index
    if index != t.cuda.current_device():
        with t.cuda.device(index):
            return ss_cache_read(cache, seq, slot, dtype, k, v, stream)
    n, kv, hd, i32 = seq.numel(), cache.n_kv_heads, cache.head_dim, t.int32
    if k is None:
        k = t.empty((n, kv, hd), dtype=dtype or t.float16, device=cache.device)
    if v is None:
        v = t.empty_like(k, memory_format=t.contiguous_format)
    _check(_lib.ss_cache_read(cache.struct, _table(seq, "seq", index, n, i32), _table(slot, "slot", index, n, i32), n, _rows(k, "k", index, kv, hd),
                              _rows(v, "v", index, kv, hd), _on(stream, index, k, v, seq, slot, *cache.tensors)))
    return k, v


def ss_tree_mask(parents, max_nodes: int) -> np.ndarray:
    """int64 [n, (max_nodes + 63) // 64] on the host: the bits of the nodes that each node of a tree sees (itself and those above it);
    parents[t] < t, -1 for a node below the history."""
    p, max_nodes = _i32(parents), _count(max_nodes, "max_nodes")
    mask = np.zeros((len(p), (max(max_nodes, 1) + 63) // 64), np.int64)
    _check(lib().ss_tree_mask(_ptr(p), len(p), max_nodes, _ptr(mask)))
    return mask


def ss_attention_tree_workspace(n_heads: int, n_kv_heads: int, head_dim: int, n_seq: int, max_context: int, max_nodes: int = 1) -> int:
    """Bytes of workspace that ss_attention_tree takes for these counts on the current device."""
    need = C.c_size_t(0)
    for n, name in ((n_heads, "n_heads"), (n_kv_heads, "n_kv_heads"), (n_seq, "n_seq"), (max_context, "max_context"), (max_nodes, "max_nodes")):
        _count(n, name)
    _check(lib().ss_attention_tree_workspace(n_heads, n_kv_heads, head_dim, n_seq, max_context, max_nodes, need))
    return need.value


def ss_attention_tree(q, cache: Cache, context, max_context: int, nodes=None, max_nodes: int = 1, mask=None, seq=None,
                      scale: Optional[float] = None, out=None, workspace=None, stream: Optional[int] = None):
    """Attention of single tokens, or of the nodes of drafted trees, over a cache that holds their own keys and values behind context[j]
    slots of history.  q [rows, heads, head_dim]; context int32 [n]; nodes int32 [n + 1] (None: a row each); mask int64
    [rows, words] as of ss_tree_mask (None: a chain); seq int32 [n] (None: sequence j).  scale: head_dim ** -0.5 if not given.
    workspace: a uint8 tensor (a new one if not given).  Returns out, a new tensor if not given (rows of no sequence are then undefined)."""
    t, index = _torch, cache.index
    if index != t.cuda.current_device():
        with t.cuda.device(index):
            return ss_attention_tree(q, cache, context, max_context, nodes, max_nodes, mask, seq, scale, out, workspace, stream)
    hd, n, i32 = cache.head_dim, context.numel(), t.int32
    _count(max_context, "max_context")
    _count(max_nodes, "max_nodes")
    qr = _rows(q, "q", index, None, hd)
    rows, heads = q.shape[0], q.shape[1]
    if out is None:
        out = t.empty_like(q, memory_format=t.contiguous_format)
    if workspace is None:
        need = C.c_size_t(0)
        _check(_lib.ss_attention_tree_workspace(heads, cache.n_kv_heads, hd, n, max_context, max_nodes, need))
        if need.value:
            workspace = t.empty(need.value, dtype=t.uint8, device=cache.device)
    size = 0 if workspace is None else workspace.numel()
    _check(_lib.ss_attention_tree(cache.struct, qr, _rows(out, "out", index, heads, hd), heads, n, _table(seq, "seq", index, n, i32),
                                  _table(context, "context", index, n, i32), max_context, _table(nodes, "nodes", index, n + 1, i32), max_nodes,
                                  _table(mask, "mask", index, rows * ((max(max_nodes, 1) + 63) // 64), t.int64), hd ** -0.5 if scale is None else scale,
                                  _table(workspace, "workspace", index, size, t.uint8), size,
                                  _on(stream, index, q, out, seq, context, nodes, mask, workspace, *cache.tensors)))
    return out


def ss_attention_packed(q, k, v, offsets, max_len: int, scale: Optional[float] = None, out=None, stream: Optional[int] = None):
    """Causal attention of packed prompts: rows offsets[i] .. offsets[i+1] - 1 (int32) are sequence i's tokens, at most max_len.  q [rows,
    heads, head_dim]; k, v [rows, kv_heads, head_dim].  Returns out, a new tensor if not given (rows of no sequence are then undefined)."""
    t, index = _with_torch(), q.get_device()
    if index < 0:
        _refuse(q, "q", index, "")
    if index != t.cuda.current_device():
        with t.cuda.device(index):
            return ss_attention_packed(q, k, v, offsets, max_len, scale, out, stream)
    _count(max_len, "max_len")
    for x, name in ((q, "q"), (k, "k")):
        if x.dim() != 3:
            _refuse(x, name, index, "[rows, heads, head_dim] of float16 or bfloat16")
    heads, hd, kv, n = q.shape[1], q.shape[2], k.shape[1], offsets.numel() - 1
    if out is None:
        out = t.empty_like(q, memory_format=t.contiguous_format)
    _check(_lib.ss_attention_packed(_rows(q, "q", index, heads, hd), _rows(k, "k", index, kv, hd), _rows(v, "v", index, kv, hd),
                                    _rows(out, "out", index, heads, hd), heads, kv, hd, _table(offsets, "offsets", index, n + 1, t.int32), n, max_len,
                                    hd ** -0.5 if scale is None else scale, _on(stream, index, q, k, v, out, offsets)))
    return out


# ---------------------------------------------------------------------------------------------------- caches in pages, beam search


class Pages:
    """The pool of pages of one layer (ss_pages): a view of tensors that the caller owns.

    k, v              flat, pages * n_kv_heads * page_slots * head_dim elements of float16, bfloat16 or int8
    k_scale, v_scale  flat float32, pages * n_kv_heads * page_slots, with int8
    """

    def __init__(self, k, v, page_slots: int, n_kv_heads: int, head_dim: int, k_scale=None, v_scale=None):
        t = _with_torch()
        if n_kv_heads < 1 or head_dim not in (64, 128) or page_slots not in (16, 32, 64, 128, 256):
            raise ValueError("n_kv_heads must be positive, head_dim 64 or 128, page_slots 16, 32, 64, 128 or 256")
        vectors = n_kv_heads * page_slots
        if k.dtype not in _ELEMENT or not k.is_cuda or k.numel() % (vectors * head_dim) or k.numel() == 0:
            _refuse(k, "k", k.get_device(), "whole pages, at least one, of float16, bfloat16 or int8")
        index, dtype, n = k.get_device(), _ELEMENT[k.dtype], k.numel() // (vectors * head_dim)
        _count(n, "the number of pages")
        if (dtype == SS_I8) != (k_scale is not None) or (dtype == SS_I8) != (v_scale is not None):
            raise ValueError("k_scale and v_scale belong to int8 pages, and only to them")
        ptr = [_table(x, name, index, k.numel(), k.dtype) for x, name in ((k, "k"), (v, "v"))]
        ptr += [_table(x, name, index, n * vectors, t.float32) for x, name in ((k_scale, "k_scale"), (v_scale, "v_scale"))]
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.page_slots, self.n_kv_heads, self.head_dim = n, page_slots, n_kv_heads, head_dim
        self.device, self.index = k.device, index
        self.struct = ss_pages(*ptr, n, page_slots, n_kv_heads, head_dim, dtype)
        self.tensors = (k, v, k_scale, v_scale)

    @classmethod
    def allocate(cls, n_pages: int, page_slots: int, n_kv_heads: int, head_dim: int, dtype, device="cuda") -> "Pages":
        """Empty pages of torch.float16, bfloat16 or int8."""
        t = _with_torch()
        if min(n_pages, page_slots, n_kv_heads, head_dim) < 1:
            raise ValueError("n_pages, page_slots, n_kv_heads and head_dim must be positive")
        vectors = n_pages * n_kv_heads * page_slots
        k, v = (t.zeros(vectors * head_dim, dtype=dtype, device=device) for _ in range(2))
        scales = [t.zeros(vectors, device=device) if dtype == t.int8 else None for _ in range(2)]
        return cls(k, v, page_slots, n_kv_heads, head_dim, *scales)


class PageTable:
    """Which pages hold the positions of each row, in every layer alike (ss_page_table): a view of tensors that the caller owns.

    pages    int32 [rows, stride]: page of positions page_slots * e .. page_slots * (e + 1) - 1 in entry e; -1: none
    lengths  int32 [rows]
    """

    def __init__(self, pages, lengths, page_slots: int, n_pages: int):
        t = _with_torch()
        if page_slots not in (16, 32, 64, 128, 256) or n_pages < 1:
            raise ValueError("page_slots must be 16, 32, 64, 128 or 256, n_pages positive")
        index = lengths.get_device()
        if index < 0:
            _refuse(lengths, "lengths", index, "")
        if pages.dim() != 2 or pages.shape[0] != lengths.numel():
            _refuse(pages, "pages", index, f"[{lengths.numel()}, entries] of {t.int32}")
        rows, stride = pages.shape
        _count(n_pages, "n_pages")
        _count(rows, "the number of rows")
        _count(stride, "the number of entries")
        self.struct = ss_page_table(_table(pages, "pages", index, rows * stride, t.int32), _table(lengths, "lengths", index, rows, t.int32),
                                    rows, stride, page_slots, n_pages)
        self.pages, self.lengths, self.page_slots, self.n_pages = pages, lengths, page_slots, n_pages
        self.rows, self.stride, self.device, self.index = rows, stride, lengths.device, index
        self.tensors = (pages, lengths)

    @classmethod
    def allocate(cls, rows: int, stride: int, page_slots: int, n_pages: int, device="cuda") -> "PageTable":
        """`rows` rows without pages, with room for `stride` each."""
        t = _with_torch()
        return cls(t.full((rows, stride), -1, dtype=t.int32, device=device), t.zeros(rows, dtype=t.int32, device=device), page_slots, n_pages)


def _same_device(index: int, *others):
    for name, x in others:
        if x.index != index:
            raise ValueError(f"{name} must be on cuda:{index}: it is on {x.device}")


def ss_pages_write(pages: Pages, table: PageTable, k, v, row=None, pos=None, stream: Optional[int] = None) -> None:
    """Keys and values [n, n_kv_heads, head_dim] of n tokens to position pos[t] of row row[t] (int32 [n]; -1: passed over); without row and
    pos, of one token per row to its last position."""
    t, index = _torch, pages.index
    if index != t.cuda.current_device():
        with t.cuda.device(index):
            return ss_pages_write(pages, table, k, v, row, pos, stream)
    _same_device(index, ("table", table))
    n, kv, hd, i32 = k.shape[0], pages.n_kv_heads, pages.head_dim, t.int32
    _check(_lib.ss_pages_write(pages.struct, table.struct, _rows(k, "k", index, kv, hd), _rows(v, "v", index, kv, hd), _table(row, "row", index, n, i32),
                               _table(pos, "pos", index, n, i32), _count(n, "the number of tokens"), _on(stream, index, k, v, row, pos, *pages.tensors, *table.tensors)))


def ss_pages_read(pages: Pages, table: PageTable, row=None, pos=None, dtype=None, k=None, v=None, stream: Optional[int] = None):
    """(k, v) [n, n_kv_heads, head_dim]: what position pos[t] of row row[t] stands for; without row and pos, the last position of each row.
    Into k and v if they are given, whose rows of tokens that do not exist stay as they are; into new tensors of `dtype` (float16)
    otherwise, where those rows are undefined."""
    t, index = _torch, pages.index
    if index != t.cuda.current_device():
        with t.cuda.device(index):
            return ss_pages_read(pages, table, row, pos, dtype, k, v, stream)
    _same_device(index, ("table", table))
    n, kv, hd, i32 = table.rows if row is None else row.numel(), pages.n_kv_heads, pages.head_dim, t.int32
    if k is None:
        k = t.empty((n, kv, hd), dtype=dtype or t.float16, device=pages.device)
    if v is None:
        v = t.empty_like(k, memory_format=t.contiguous_format)
    _check(_lib.ss_pages_read(pages.struct, table.struct, _table(row, "row", index, n, i32), _table(pos, "pos", index, n, i32), _count(n, "the number of tokens"),
                              _rows(k, "k", index, kv, hd), _rows(v, "v", index, kv, hd), _on(stream, index, k, v, row, pos, *pages.tensors, *table.tensors)))
    return k, v


def ss_attention_pages_workspace(n_heads: int, n_kv_heads: int, head_dim: int, page_slots: int, stride: int, n: int, max_length: int,
                                 group: int = 1) -> int:
    """Bytes of workspace that ss_attention_pages takes for these counts, and a table of `stride` entries a row, on the current device."""
    need = C.c_size_t(0)
    for x, name in ((n_heads, "n_heads"), (n_kv_heads, "n_kv_heads"), (stride, "stride"), (n, "n"), (max_length, "max_length"), (group, "group")):
        _count(x, name)
    _check(lib().ss_attention_pages_workspace(n_heads, n_kv_heads, head_dim, page_slots, stride, n, max_length, group, need))
    return need.value


def ss_attention_pages(q, pages: Pages, table: PageTable, max_length: int, group: int = 1, rows=None, scale: Optional[float] = None, out=None,
                       workspace=None, stream: Optional[int] = None):
    """Attention of one token per row, q [n, heads, head_dim], over the pages of its row of the table (rows int32 [n]; None: row j), which
    hold its own key and value too.  Queries j * group .. are looked at together: pages that their rows share are read once.  scale: head_dim
    ** -0.5 if not given.  workspace: a uint8 tensor (a new one if not given).  Returns out, a new tensor if not given."""
    t, index = _torch, pages.index
    if index != t.cuda.current_device():
        with t.cuda.device(index):
            return ss_attention_pages(q, pages, table, max_length, group, rows, scale, out, workspace, stream)
    _same_device(index, ("table", table))
    hd, n = pages.head_dim, q.shape[0]
    _count(n, "the number of rows")
    _count(max_length, "max_length")
    _count(group, "group")
    qr = _rows(q, "q", index, None, hd)
    heads = q.shape[1]
    if out is None:
        out = t.empty_like(q, memory_format=t.contiguous_format)
    if workspace is None:
        need = C.c_size_t(0)
        _check(_lib.ss_attention_pages_workspace(heads, pages.n_kv_heads, hd, pages.page_slots, table.stride, n, max_length, group, need))
        if need.value:
            workspace = t.empty(need.value, dtype=t.uint8, device=pages.device)
    size = 0 if workspace is None else workspace.numel()
    _check(_lib.ss_attention_pages(pages.struct, table.struct, qr, _rows(out, "out", index, heads, hd), heads, n, _table(rows, "rows", index, n, t.int32),
                                   max_length, group, hd ** -0.5 if scale is None else scale, _table(workspace, "workspace", index, size, t.uint8), size,
                                   _on(stream, index, q, out, rows, workspace, *pages.tensors, *table.tensors)))
    return out


def ss_pages_workspace(n_pages: int) -> int:
    """Bytes of workspace that ss_pages_fork and ss_pages_compact take."""
    need = C.c_size_t(0)
    _check(lib().ss_pages_workspace(_count(n_pages, "n_pages"), need))
    return need.value


def ss_pages_fork(table: PageTable, to: PageTable, parent=None, grow=None, held=None, src=None, dst=None, missing=None, workspace=None,
                  stream: Optional[int] = None):
    """Row i of `to` takes over the pages of row parent[i] of `table` (int32 [to.rows]; None: row i; -1: none) and grows by grow[i] positions (int32; None: 1
    where there is a parent).  held uint8 [n_pages]: nonzero, somebody else holds the page too.  Returns (src, dst, missing), int32, new tensors if not
    given: the pages that ss_pages_copy has to copy for each row, -1 for none, and how many pages there were too few."""
    t, index = _torch, table.index
    if index != t.cuda.current_device():
        with t.cuda.device(index):
            return ss_pages_fork(table, to, parent, grow, held, src, dst, missing, workspace, stream)
    _same_device(index, ("to", to))
    n, i32 = to.rows, t.int32
    if src is None:
        src = t.empty(n, dtype=i32, device=table.device)
    if dst is None:
        dst = t.empty(n, dtype=i32, device=table.device)
    if missing is None:
        missing = t.empty(1, dtype=i32, device=table.device)
    if workspace is None:
        workspace = t.empty(8 * table.n_pages, dtype=t.uint8, device=table.device)
    size = workspace.numel()
    _check(_lib.ss_pages_fork(table.struct, to.struct, _table(parent, "parent", index, n, i32), _table(grow, "grow", index, n, i32),
                              _table(held, "held", index, table.n_pages, t.uint8), _table(src, "src", index, n, i32), _table(dst, "dst", index, n, i32),
                              _table(missing, "missing", index, 1, i32), _table(workspace, "workspace", index, size, t.uint8), size,
                              _on(stream, index, parent, grow, held, src, dst, missing, workspace, *table.tensors, *to.tensors)))
    return src, dst, missing


def ss_pages_compact(table: PageTable, to: Optional[PageTable] = None, held=None, src=None, dst=None, place=None, counts=None, workspace=None,
                     stream: Optional[int] = None):
    """The pages in use get the numbers 0 .. counts[0] - 1, in `to` (None: in the table itself).  Returns (src, dst, place, counts), int32, new tensors if not
    given: the pages to copy (ss_pages_copy with counts[1:]), the new number of every page (-1: free), and how many are in use and move."""
    t, index = _torch, table.index
    if index != t.cuda.current_device():
        with t.cuda.device(index):
            return ss_pages_compact(table, to, held, src, dst, place, counts, workspace, stream)
    if to is None:
        to = table
    _same_device(index, ("to", to))
    n, i32 = table.n_pages, t.int32
    if src is None:
        src = t.empty(n // 2, dtype=i32, device=table.device)
    if dst is None:
        dst = t.empty(n // 2, dtype=i32, device=table.device)
    if place is None:
        place = t.empty(n, dtype=i32, device=table.device)
    if counts is None:
        counts = t.empty(2, dtype=i32, device=table.device)
    if workspace is None:
        workspace = t.empty(8 * n, dtype=t.uint8, device=table.device)
    size = workspace.numel()
    _check(_lib.ss_pages_compact(table.struct, to.struct, _table(held, "held", index, n, t.uint8), _table(src, "src", index, n // 2, i32),
                                 _table(dst, "dst", index, n // 2, i32), _table(place, "place", index, n, i32), _table(counts, "counts", index, 2, i32),
                                 _table(workspace, "workspace", index, size, t.uint8), size,
                                 _on(stream, index, held, src, dst, place, counts, workspace, *table.tensors, *to.tensors)))
    return src, dst, place, counts


def ss_pages_copy(layers: Sequence[Pages], src, dst, count=None, stream: Optional[int] = None) -> None:
    """Page src[i] to page dst[i] (int32 [n]; -1: passed over) in every layer, for i below count[0] if `count` (int32 [1]) is given."""
    if not layers:
        return
    t, index = _torch, layers[0].index
    if index != t.cuda.current_device():
        with t.cuda.device(index):
            return ss_pages_copy(layers, src, dst, count, stream)
    for x in layers:
        if x.index != index:
            raise ValueError(f"every layer must be on cuda:{index}: one is on {x.device}")
    n, i32 = src.numel(), t.int32
    structs = (ss_pages * len(layers))(*[x.struct for x in layers])
    _check(_lib.ss_pages_copy(structs, len(layers), _table(src, "src", index, n, i32), _table(dst, "dst", index, n, i32), _count(n, "the number of pairs"),
                              _table(count, "count", index, 1, i32),
                              _stream(index) if stream is None else _on(stream, index, src, dst, count, *(y for x in layers for y in x.tensors))))


class Beams(NamedTuple):
    """What ss_beam_select returns: the candidates that were taken, `keep` of each group."""
    parent: object    # int32 [groups * keep]: the row that each continues (ss_pages_fork's parent), -1: none
    token: object     # int32 [groups * keep]
    totals: object    # float32 [groups, keep]
    lengths: object   # int32 [groups * keep], None without lengths
    ended: object     # uint8 [groups * keep]
    history: object   # int32 [groups * keep, width], None without histories


def ss_beam_select_workspace(n_groups: int, beams: int, vocab: int, keep: int) -> int:
    """Bytes of workspace that ss_beam_select takes."""
    need = C.c_size_t(0)
    for x, name in ((n_groups, "n_groups"), (beams, "beams"), (vocab, "vocab"), (keep, "keep")):
        _count(x, name)
    _check(lib().ss_beam_select_workspace(n_groups, beams, vocab, keep, need))
    return need.value


def ss_beam_select(logits, totals, keep: int, lengths=None, ended=None, end_id: int = -1, length_power: float = 0.0, history=None, out: Optional[Beams] = None,
                   workspace=None, stream: Optional[int] = None) -> Beams:
    """A step of beam search: of all continuations of the beams of each group the `keep` best, by the sum of their tokens' log probabilities over
    length ** length_power.  logits [groups * beams, vocab] of float32, float16 or bfloat16; totals float32 [groups, beams]; lengths int32 and ended uint8
    [groups * beams]; history int32 [groups * beams, width].  Returns the new state in new tensors, or in `out`'s."""
    t = _with_torch()
    index = logits.get_device()
    if index < 0:
        _refuse(logits, "logits", index, "")
    if index != t.cuda.current_device():
        with t.cuda.device(index):
            return ss_beam_select(logits, totals, keep, lengths, ended, end_id, length_power, history, out, workspace, stream)
    for x, name in ((logits, "logits"), (totals, "totals")):
        if x.requires_grad and t.is_grad_enabled():
            raise ValueError(f"{name} requires gradients, and this operator has none: call it under torch.no_grad(), or with {name}.detach()")
    dtype = SS_F32 if logits.dtype is t.float32 else _ELEMENT.get(logits.dtype, SS_I8)
    if totals.dim() != 2:
        _refuse(totals, "totals", index, "[groups, beams] of float32")
    groups, beams = totals.shape
    if logits.dim() != 2 or logits.shape[0] != groups * beams or dtype == SS_I8 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        _refuse(logits, "logits", index, f"[{groups * beams}, vocab] of float32, float16 or bfloat16 whose last dimension is contiguous")
    for x, name in ((keep, "keep"), (end_id, "end_id"), (logits.shape[0], "the number of rows"), (logits.shape[1], "vocab")):
        _count(x, name)
    vocab, rows, n, i32, dev = logits.shape[1], groups * beams, groups * max(keep, 0), t.int32, logits.device
    if history is not None and (history.dim() != 2 or history.shape[0] != rows):
        _refuse(history, "history", index, f"[{rows}, width] of int32")
    width = 0 if history is None else history.shape[1]
    if out is None:
        out = Beams(t.empty(n, dtype=i32, device=dev), t.empty(n, dtype=i32, device=dev), t.empty((groups, max(keep, 0)), dtype=t.float32, device=dev),
                    None if lengths is None else t.empty(n, dtype=i32, device=dev), t.empty(n, dtype=t.uint8, device=dev),
                    None if history is None else t.empty((n, width), dtype=i32, device=dev))
    if out.history is not None and (out.history.dim() != 2 or out.history.shape[0] != n):
        _refuse(out.history, "out.history", index, f"[{n}, width] of int32")
    new_width = 0 if out.history is None else out.history.shape[1]
    _count(max(width, new_width), "the width of histories")
    now = ss_beams(_table(totals, "totals", index, rows, t.float32), _table(lengths, "lengths", index, rows, i32), _table(ended, "ended", index, rows, t.uint8),
                   _table(history, "history", index, rows * width, i32), width)
    to = ss_beams(_table(out.totals, "out.totals", index, n, t.float32), _table(out.lengths, "out.lengths", index, n, i32),
                  _table(out.ended, "out.ended", index, n, t.uint8), _table(out.history, "out.history", index, n * new_width, i32), new_width)
    if workspace is None:
        need = C.c_size_t(0)
        _check(_lib.ss_beam_select_workspace(groups, beams, vocab, keep, need))
        workspace = t.empty(need.value, dtype=t.uint8, device=dev)
    size = workspace.numel()
    _check(_lib.ss_beam_select(logits.data_ptr(), dtype, logits.stride(0), groups, beams, vocab, keep, now, to, _table(out.parent, "out.parent", index, n, i32),
                               _table(out.token, "out.token", index, n, i32), end_id, length_power, _table(workspace, "workspace", index, size, t.uint8), size,
                               _on(stream, index, logits, totals, lengths, ended, history, workspace, *out)))
    return out

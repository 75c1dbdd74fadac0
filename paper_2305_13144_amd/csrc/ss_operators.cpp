// C ABI of the operators on device tensors: argument checks and launches.  They run on the caller's stream and return once
// enqueued; they allocate nothing and wait for nothing, so a caller may capture them into a graph.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>

#include "ss_internal.h"
#include "ss_kernels.h"

namespace {

using ss::fail;

static_assert(ss::kBF16 == SS_BF16 && ss::kF16 == SS_F16 && ss::kI8 == SS_I8, "element types");

bool is_half(int32_t dtype) { return dtype == SS_F16 || dtype == SS_BF16; }
bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

int check_cache(const ss_cache* c)
{
    if (!c) return fail(SS_EINVAL, "cache is NULL");
    if (c->head_dim != 64 && c->head_dim != 128) return fail(SS_EINVAL, "cache: head_dim must be 64 or 128");
    if (!is_half(c->dtype) && c->dtype != SS_I8) return fail(SS_EINVAL, "cache: dtype must be SS_F16, SS_BF16 or SS_I8");
    if (c->n_kv_heads > 65535) return fail(SS_EINVAL, "cache: more than 65535 heads");
    if (c->n_seq < 0 || c->n_kv_heads < 1 || c->total_slots < 0) return fail(SS_EINVAL, "cache: bad number of sequences, heads or slots");
    if (c->total_slots > 0 && (!c->k || !c->v)) return fail(SS_EINVAL, "cache: k or v is NULL");
    if (!aligned(c->k) || !aligned(c->v)) return fail(SS_EINVAL, "cache: k and v must be 16-byte aligned");
    if (c->dtype == SS_I8 && c->total_slots > 0 && (!c->k_scale || !c->v_scale)) return fail(SS_EINVAL, "cache: SS_I8 needs k_scale and v_scale");
    if (c->n_seq > 0 && (!c->start || !c->slots)) return fail(SS_EINVAL, "cache: start or slots is NULL");
    return SS_OK;
}

int check_rows(const ss_rows* r, const char* name)
{
    if (!r) return fail(SS_EINVAL, "%s is NULL", name);
    if (!is_half(r->dtype)) return fail(SS_EINVAL, "%s: dtype must be SS_F16 or SS_BF16", name);
    if (r->rows < 0) return fail(SS_EINVAL, "%s: negative number of rows", name);
    if (r->rows > 0 && !r->p) return fail(SS_EINVAL, "%s: NULL pointer", name);
    if (r->row_stride < 0 || r->head_stride < 0 || r->row_stride > (1 << 24) || r->head_stride > (1ll << 40))
        return fail(SS_EINVAL, "%s: strides must be 0 to 2^24 (rows) and 2^40 (heads)", name);
    if (!aligned(r->p) || r->row_stride % 8 || r->head_stride % 8)
        return fail(SS_EINVAL, "%s must be 16-byte aligned, its strides multiples of 8 elements", name);
    return SS_OK;
}

// Rows that are written: no two heads of any two rows share an element, in the order [rows][heads] or [heads][rows].
int check_apart(const ss_rows* r, const char* name, int64_t n_heads, int32_t head_dim)
{
    const bool by_rows = (n_heads == 1 || r->head_stride >= head_dim) && (r->rows < 2 || r->row_stride >= (n_heads - 1) * r->head_stride + head_dim);
    const bool by_heads = (r->rows < 2 || r->row_stride >= head_dim) && (n_heads == 1 || r->head_stride >= (r->rows - 1) * r->row_stride + head_dim);
    return by_rows || by_heads ? SS_OK : fail(SS_EINVAL, "%s: its rows overlap", name);
}

ss::CacheView view(const ss_cache* c)
{
    return {c->k, c->v, c->k_scale, c->v_scale, c->start, c->slots, c->total_slots, c->n_seq, c->n_kv_heads, c->head_dim, c->dtype};
}
ss::RowsView view(const ss_rows* r) { return {r->p, r->row_stride, r->head_stride, r->rows}; }

// Runs f, which launches, and says what became of it.  An error that an earlier call of the caller's left behind is not this call's.
template <class F>
int launch(F f)
{
    (void)hipGetLastError();
    f();
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SS_OK : fail(SS_EDEVICE, "launch failed: %s", hipGetErrorString(e));
}

// Compute units of the current device, asked for once per device (256 where there is none to ask).
int compute_units()
{
    static std::atomic<int> known[64];
    int device = 0, n = 0;
    if (hipGetDevice(&device) != hipSuccess || device < 0 || device >= 64) {
        (void)hipGetLastError();
        return 256;
    }
    n = known[device].load(std::memory_order_relaxed);
    if (n > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess || n < 1) {
        (void)hipGetLastError();
        return 256;
    }
    known[device].store(n, std::memory_order_relaxed);
    return n;
}

int check_token_list(const ss_cache* c, const ss_rows* k, const ss_rows* v, const int32_t* seq, const int32_t* slot, int32_t n)
{
    if (int rc = check_cache(c)) return rc;
    if (int rc = check_rows(k, "k")) return rc;
    if (int rc = check_rows(v, "v")) return rc;
    if (n < 0) return fail(SS_EINVAL, "negative number of tokens");
    if (k->dtype != v->dtype) return fail(SS_EINVAL, "k and v differ in type");
    if (k->rows < n || v->rows < n) return fail(SS_EINVAL, "k and v have fewer than %d rows", n);
    if (n > 0 && (!seq || !slot)) return fail(SS_EINVAL, "seq or slot is NULL");
    // workgroups of 256 threads take 16 tokens each, and a grid has fewer than 2^32 threads a dimension
    if (n > SS_CACHE_MAX_TOKENS) return fail(SS_EINVAL, "more than %d tokens", SS_CACHE_MAX_TOKENS);
    if ((int64_t)n * c->n_kv_heads > INT_MAX) return fail(SS_EINVAL, "more than 2^31 vectors");
    return SS_OK;
}

int check_tree_counts(int32_t n_heads, int32_t n_kv_heads, int32_t n_seq, int32_t max_context, int32_t max_nodes)
{
    if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads) return fail(SS_EINVAL, "n_heads must be a multiple of the key/value heads");
    if (n_heads > 65535) return fail(SS_EINVAL, "more than 65535 heads");
    if (n_seq < 0 || max_context < 0) return fail(SS_EINVAL, "negative number of sequences or context");
    if (n_seq > 65535) return fail(SS_EINVAL, "more than 65535 sequences");
    if (max_nodes < 1 || max_nodes > SS_TREE_MAX_NODES) return fail(SS_EINVAL, "max_nodes must be 1 to %d", SS_TREE_MAX_NODES);
    if (max_context > INT_MAX - SS_TREE_MAX_NODES - 256) return fail(SS_EINVAL, "max_context is too large");
    if ((int64_t)n_seq * n_heads * max_nodes > INT_MAX / 4) return fail(SS_EINVAL, "too many rows");
    return SS_OK;
}

ss::TreePlan plan_of(int32_t n_heads, int32_t n_kv_heads, int32_t n_seq, int32_t max_context, int32_t max_nodes)
{
    return ss::tree_plan(n_seq, n_kv_heads, max_nodes * (n_heads / n_kv_heads), max_context + max_nodes, compute_units());
}

size_t part_bytes(const ss::TreePlan& p, int32_t n_heads, int32_t head_dim, int32_t n_seq, int32_t max_nodes)
{
    return p.chunks > 1 ? (size_t)n_seq * p.chunks * max_nodes * n_heads * (head_dim + 4) * 4 : 0;
}

}  // namespace

extern "C" int ss_cache_write(const ss_cache* cache, const ss_rows* k, const ss_rows* v, const int32_t* seq, const int32_t* slot, int32_t n,
                              void* hip_stream)
{
    ss::clear_error();
    if (int rc = check_token_list(cache, k, v, seq, slot, n)) return rc;
    if (n == 0 || cache->n_seq == 0) return SS_OK;
    return launch([&] { ss::launch_cache_write(view(cache), view(k), view(v), k->dtype, seq, slot, n, (hipStream_t)hip_stream); });
}

extern "C" int ss_cache_read(const ss_cache* cache, const int32_t* seq, const int32_t* slot, int32_t n, const ss_rows* k, const ss_rows* v,
                             void* hip_stream)
{
    ss::clear_error();
    if (int rc = check_token_list(cache, k, v, seq, slot, n)) return rc;
    if (int rc = check_apart(k, "k", cache->n_kv_heads, cache->head_dim)) return rc;
    if (int rc = check_apart(v, "v", cache->n_kv_heads, cache->head_dim)) return rc;
    if (n == 0 || cache->n_seq == 0) return SS_OK;
    return launch([&] { ss::launch_cache_read(view(cache), view(k), view(v), k->dtype, seq, slot, n, (hipStream_t)hip_stream); });
}

extern "C" int ss_attention_tree_workspace(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t n_seq, int32_t max_context,
                                           int32_t max_nodes, size_t* bytes)
{
    ss::clear_error();
    if (!bytes) return fail(SS_EINVAL, "bytes is NULL");
    if (head_dim != 64 && head_dim != 128) return fail(SS_EINVAL, "head_dim must be 64 or 128");
    if (int rc = check_tree_counts(n_heads, n_kv_heads, n_seq, max_context, max_nodes)) return rc;
    *bytes = part_bytes(plan_of(n_heads, n_kv_heads, n_seq, max_context, max_nodes), n_heads, head_dim, n_seq, max_nodes);
    return SS_OK;
}

extern "C" int ss_attention_tree(const ss_cache* cache, const ss_rows* q, const ss_rows* out, int32_t n_heads, int32_t n_seq,
                                 const int32_t* seq, const int32_t* context, int32_t max_context, const int32_t* nodes, int32_t max_nodes,
                                 const uint64_t* mask, float scale, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    ss::clear_error();
    if (int rc = check_cache(cache)) return rc;
    if (int rc = check_rows(q, "q")) return rc;
    if (int rc = check_rows(out, "out")) return rc;
    if (int rc = check_tree_counts(n_heads, cache->n_kv_heads, n_seq, max_context, max_nodes)) return rc;
    if (q->dtype != out->dtype) return fail(SS_EINVAL, "q and out differ in type");
    if (cache->dtype != SS_I8 && cache->dtype != q->dtype) return fail(SS_EINVAL, "a cache of 16 bits and q must have the same type");
    if (out->rows < q->rows) return fail(SS_EINVAL, "out has fewer rows than q");
    if (!std::isfinite(scale)) return fail(SS_EINVAL, "scale must be finite");
    if (int rc = check_apart(out, "out", n_heads, cache->head_dim)) return rc;
    if (!nodes && max_nodes != 1) return fail(SS_EINVAL, "nodes is NULL: max_nodes must be 1");
    if (!nodes && q->rows < n_seq) return fail(SS_EINVAL, "q has fewer than %d rows", n_seq);
    if (!seq && n_seq > cache->n_seq) return fail(SS_EINVAL, "the cache has fewer than %d sequences", n_seq);
    if (n_seq > 0 && !context) return fail(SS_EINVAL, "context is NULL");
    if (n_seq == 0 || q->rows == 0) return SS_OK;
    if (cache->n_seq == 0) return fail(SS_EINVAL, "the cache has no sequences");
    const ss::TreePlan p = plan_of(n_heads, cache->n_kv_heads, n_seq, max_context, max_nodes);
    const size_t need = part_bytes(p, n_heads, cache->head_dim, n_seq, max_nodes);
    if (need > workspace_bytes || (need > 0 && !workspace))
        return fail(SS_EINVAL, "this call needs %zu bytes of workspace, it was given %zu", need, workspace ? workspace_bytes : (size_t)0);
    if (need > 0 && !aligned(workspace)) return fail(SS_EINVAL, "workspace must be 16-byte aligned");
    ss::TreeArgs a{};
    a.c = view(cache);
    a.q = view(q);
    a.out = view(out);
    a.seq = seq;
    a.context = context;
    a.nodes = nodes;
    a.mask = mask;
    a.part = (float*)workspace;
    a.scale = scale;
    a.n_seq = n_seq;
    a.heads = n_heads;
    a.max_nodes = max_nodes;
    a.words = (max_nodes + 63) / 64;
    a.chunk = p.chunk;
    a.chunks = p.chunks;
    a.row_blocks = p.row_blocks;
    return launch([&] { ss::launch_attention_tree(a, q->dtype, p.tiles, (hipStream_t)hip_stream); });
}

extern "C" int ss_tree_mask(const int32_t* parents, int32_t n, int32_t max_nodes, uint64_t* mask)
{
    ss::clear_error();
    if (n < 0 || (n > 0 && (!parents || !mask))) return fail(SS_EINVAL, "NULL or negative argument");
    if (max_nodes < 1 || max_nodes > SS_TREE_MAX_NODES) return fail(SS_EINVAL, "max_nodes must be 1 to %d", SS_TREE_MAX_NODES);
    if (n > max_nodes) return fail(SS_EINVAL, "a tree of %d nodes, max_nodes is %d", n, max_nodes);
    for (int32_t t = 0; t < n; ++t)
        if (parents[t] < -1 || parents[t] >= t) return fail(SS_EINVAL, "parents[%d] must be -1 or an earlier node", t);
    ss::tree_mask(parents, n, (max_nodes + 63) / 64, mask);
    return SS_OK;
}

extern "C" int ss_attention_packed(const ss_rows* q, const ss_rows* k, const ss_rows* v, const ss_rows* out, int32_t n_heads,
                                   int32_t n_kv_heads, int32_t head_dim, const int32_t* offsets, int32_t n_seq, int32_t max_len, float scale,
                                   void* hip_stream)
{
    ss::clear_error();
    if (int rc = check_rows(q, "q")) return rc;
    if (int rc = check_rows(k, "k")) return rc;
    if (int rc = check_rows(v, "v")) return rc;
    if (int rc = check_rows(out, "out")) return rc;
    if (head_dim != 64 && head_dim != 128) return fail(SS_EINVAL, "head_dim must be 64 or 128");
    if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads) return fail(SS_EINVAL, "n_heads must be a multiple of the key/value heads");
    if (q->dtype != k->dtype || q->dtype != v->dtype || q->dtype != out->dtype) return fail(SS_EINVAL, "q, k, v and out differ in type");
    if (k->rows < q->rows || v->rows < q->rows || out->rows < q->rows) return fail(SS_EINVAL, "k, v or out has fewer rows than q");
    if (n_heads > 65535) return fail(SS_EINVAL, "more than 65535 heads");
    if (n_seq < 0 || max_len < 0) return fail(SS_EINVAL, "negative number of sequences or length");
    if (!std::isfinite(scale)) return fail(SS_EINVAL, "scale must be finite");
    if (int rc = check_apart(out, "out", n_heads, head_dim)) return rc;
    if (n_seq > 65535) return fail(SS_EINVAL, "more than 65535 sequences");
    if (max_len > 64 * 65535) return fail(SS_EINVAL, "max_len is too large");
    if (n_seq == 0 || max_len == 0 || q->rows == 0) return SS_OK;
    if (!offsets) return fail(SS_EINVAL, "offsets is NULL");
    ss::PackedArgs a{};
    a.q = view(q);
    a.k = view(k);
    a.v = view(v);
    a.out = view(out);
    a.offsets = offsets;
    a.scale = scale;
    a.heads = n_heads;
    a.n_kv = n_kv_heads;
    a.max_len = (int32_t)std::min<int64_t>(max_len, q->rows);   // no sequence is longer: no workgroups for what a caller only allows
    return launch([&] { ss::launch_attention_packed(a, head_dim, q->dtype, n_seq, (hipStream_t)hip_stream); });
}

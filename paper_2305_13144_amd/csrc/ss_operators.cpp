// C ABI of the operators on device tensors: argument checks and launches.  They run on the caller's stream and return once
// enqueued; they allocate nothing and wait for nothing, so a caller may capture them into a graph.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>
#include <vector>

#include "ss_internal.h"
#include "ss_kernels.h"

namespace {

using ss::fail;

static_assert(ss::kBF16 == SS_BF16 && ss::kF32 == SS_F32 && ss::kF16 == SS_F16 && ss::kI8 == SS_I8, "element types");
static_assert(ss::kBeamMax == SS_BEAM_MAX, "beams");

bool is_half(int32_t dtype) { return dtype == SS_F16 || dtype == SS_BF16; }
bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool is_page_size(int32_t n) { return n == 16 || n == 32 || n == 64 || n == 128 || n == 256; }

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

int check_pages(const ss_pages* p)
{
    if (!p) return fail(SS_EINVAL, "pages is NULL");
    if (p->head_dim != 64 && p->head_dim != 128) return fail(SS_EINVAL, "pages: head_dim must be 64 or 128");
    if (!is_half(p->dtype) && p->dtype != SS_I8) return fail(SS_EINVAL, "pages: dtype must be SS_F16, SS_BF16 or SS_I8");
    if (p->n_kv_heads < 1 || p->n_kv_heads > 65535) return fail(SS_EINVAL, "pages: 1 to 65535 heads");
    if (p->n_pages < 1 || p->n_pages > SS_PAGES_MAX) return fail(SS_EINVAL, "pages: there must be a page, and at most %d pages", SS_PAGES_MAX);
    if (!is_page_size(p->page_slots)) return fail(SS_EINVAL, "pages: page_slots must be 16, 32, 64, 128 or 256");
    if (!p->k || !p->v) return fail(SS_EINVAL, "pages: k or v is NULL");
    if (!aligned(p->k) || !aligned(p->v)) return fail(SS_EINVAL, "pages: k and v must be 16-byte aligned");
    if (p->dtype == SS_I8 && (!p->k_scale || !p->v_scale)) return fail(SS_EINVAL, "pages: SS_I8 needs k_scale and v_scale");
    if (p->dtype == SS_I8 && (!aligned(p->k_scale) || !aligned(p->v_scale))) return fail(SS_EINVAL, "pages: k_scale and v_scale must be 16-byte aligned");
    return SS_OK;
}

int check_table(const ss_page_table* t, const char* name)
{
    if (!t) return fail(SS_EINVAL, "%s is NULL", name);
    if (t->n_rows < 0 || t->stride < 0) return fail(SS_EINVAL, "%s: negative number of rows or entries", name);
    if (t->n_pages < 1 || t->n_pages > SS_PAGES_MAX) return fail(SS_EINVAL, "%s: there must be a page, and at most %d pages", name, SS_PAGES_MAX);
    if (!is_page_size(t->page_slots)) return fail(SS_EINVAL, "%s: page_slots must be 16, 32, 64, 128 or 256", name);
    if ((int64_t)t->stride * t->page_slots > INT_MAX - 1024) return fail(SS_EINVAL, "%s: rows of more than 2^31 positions", name);
    if ((int64_t)t->n_rows * t->stride > INT_MAX) return fail(SS_EINVAL, "%s: more than 2^31 entries", name);
    if (t->n_rows > 0 && (!t->lengths || (t->stride > 0 && !t->pages))) return fail(SS_EINVAL, "%s: pages or lengths is NULL", name);
    return SS_OK;
}

int check_pages_and_table(const ss_pages* p, const ss_page_table* t)
{
    if (int rc = check_pages(p)) return rc;
    if (int rc = check_table(t, "table")) return rc;
    if (t->page_slots != p->page_slots || t->n_pages != p->n_pages) return fail(SS_EINVAL, "table and pages differ in page_slots or n_pages");
    return SS_OK;
}

int check_page_tokens(const ss_pages* p, const ss_page_table* t, const ss_rows* k, const ss_rows* v, const int32_t* row, const int32_t* pos, int32_t n)
{
    if (int rc = check_pages_and_table(p, t)) return rc;
    if (int rc = check_rows(k, "k")) return rc;
    if (int rc = check_rows(v, "v")) return rc;
    if (n < 0) return fail(SS_EINVAL, "negative number of tokens");
    if (k->dtype != v->dtype) return fail(SS_EINVAL, "k and v differ in type");
    if (k->rows < n || v->rows < n) return fail(SS_EINVAL, "k and v have fewer than %d rows", n);
    if (!row != !pos) return fail(SS_EINVAL, "row and pos are given together or not at all");
    if (n > SS_CACHE_MAX_TOKENS) return fail(SS_EINVAL, "more than %d tokens", SS_CACHE_MAX_TOKENS);
    if ((int64_t)n * p->n_kv_heads > INT_MAX) return fail(SS_EINVAL, "more than 2^31 vectors");
    return SS_OK;
}

int check_two_tables(const ss_page_table* from, const ss_page_table* to)
{
    if (int rc = check_table(from, "from")) return rc;
    if (int rc = check_table(to, "to")) return rc;
    if (from->page_slots != to->page_slots || from->n_pages != to->n_pages) return fail(SS_EINVAL, "from and to differ in page_slots or n_pages");
    if (from->n_rows > SS_PAGES_MAX_ROWS || to->n_rows > SS_PAGES_MAX_ROWS) return fail(SS_EINVAL, "more than %d rows", SS_PAGES_MAX_ROWS);
    return SS_OK;
}

// Whether a part of one table is in the other; `in_place`: other than the same part in the same place.
bool tables_meet(const ss_page_table* a, const ss_page_table* b, bool in_place)
{
    struct Part {
        const void* p;
        size_t bytes;
    };
    auto parts = [](const ss_page_table* t, Part (&of)[2]) {
        of[0] = {t->pages, (size_t)t->n_rows * t->stride * 4};
        of[1] = {t->lengths, (size_t)t->n_rows * 4};
    };
    Part x[2], y[2];
    parts(a, x);
    parts(b, y);
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) {
            const uintptr_t p = (uintptr_t)x[i].p, q = (uintptr_t)y[j].p;
            if (x[i].bytes == 0 || y[j].bytes == 0 || p >= q + y[j].bytes || q >= p + x[i].bytes) continue;
            if (!in_place || i != j || p != q) return true;
        }
    return false;
}

size_t pages_workspace(int32_t n_pages) { return (size_t)n_pages * 8; }

int check_workspace(const void* workspace, size_t given, size_t need)
{
    if (need > given || (need > 0 && !workspace))
        return fail(SS_EINVAL, "this call needs %zu bytes of workspace, it was given %zu", need, workspace ? given : (size_t)0);
    if (need > 0 && !aligned(workspace)) return fail(SS_EINVAL, "workspace must be 16-byte aligned");
    return SS_OK;
}

ss::PagesView view(const ss_pages* p) { return {p->k, p->v, p->k_scale, p->v_scale, p->n_pages, p->page_slots, p->n_kv_heads, p->head_dim, p->dtype}; }
ss::TableView view(const ss_page_table* t) { return {t->pages, t->lengths, t->n_rows, t->stride, t->page_slots, t->n_pages}; }

int check_page_attention(int32_t n_heads, int32_t n_kv_heads, int32_t page_slots, int32_t stride, int32_t n, int32_t max_length, int32_t group)
{
    if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads) return fail(SS_EINVAL, "n_heads must be a multiple of the key/value heads");
    if (n_heads > 65535) return fail(SS_EINVAL, "more than 65535 heads");
    if (n < 0 || max_length < 0) return fail(SS_EINVAL, "negative number of rows or length");
    if (n > 65535) return fail(SS_EINVAL, "more than 65535 rows");
    if (group < 1 || group > SS_PAGES_MAX_GROUP) return fail(SS_EINVAL, "group must be 1 to %d", SS_PAGES_MAX_GROUP);
    if (n % group) return fail(SS_EINVAL, "%d rows are no whole groups of %d", n, group);
    if ((int64_t)group * stride * page_slots / 16 > INT_MAX) return fail(SS_EINVAL, "the rows of a group have more than 2^31 pieces of 16 positions");
    if ((int64_t)n / group * n_kv_heads * (((int64_t)group * (n_heads / n_kv_heads) + 15) / 16) > 1 << 22) return fail(SS_EINVAL, "too many rows and heads");
    return SS_OK;
}

// No row is longer than its entries, whatever a caller allows for.
ss::PagePlan plan_of_pages(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t page_slots, int32_t stride, int32_t n, int32_t max_length, int32_t group)
{
    return ss::page_plan(n, group, n_kv_heads, n_heads / n_kv_heads, head_dim, (int)std::min<int64_t>(max_length, (int64_t)stride * page_slots), compute_units());
}

int check_beams(int32_t n_groups, int32_t beams, int32_t vocab, int32_t keep)
{
    if (beams < 1 || beams > SS_BEAM_MAX) return fail(SS_EINVAL, "beams must be 1 to %d", SS_BEAM_MAX);
    if (keep < 1 || keep > SS_BEAM_MAX) return fail(SS_EINVAL, "keep must be 1 to %d", SS_BEAM_MAX);
    if (vocab < 1) return fail(SS_EINVAL, "vocab must be positive");
    if (n_groups < 0 || (int64_t)n_groups * beams > 65535) return fail(SS_EINVAL, "0 to 65535 rows of beams");
    return SS_OK;
}

// Whatever the logits' type is: that of 32 bits has the most slices.
size_t beam_workspace(int32_t n_groups, int32_t beams, int32_t vocab, int32_t keep)
{
    return (size_t)n_groups * beams * ss::beam_slices(n_groups, beams, vocab, keep, 4, compute_units()) * ss::beam_part_floats(keep) * 4;
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

extern "C" int ss_pages_write(const ss_pages* pages, const ss_page_table* table, const ss_rows* k, const ss_rows* v, const int32_t* row,
                              const int32_t* pos, int32_t n, void* hip_stream)
{
    ss::clear_error();
    if (int rc = check_page_tokens(pages, table, k, v, row, pos, n)) return rc;
    if (n == 0 || table->n_rows == 0 || table->stride == 0) return SS_OK;
    return launch([&] { ss::launch_pages_write(view(pages), view(table), view(k), view(v), k->dtype, row, pos, n, (hipStream_t)hip_stream); });
}

extern "C" int ss_pages_read(const ss_pages* pages, const ss_page_table* table, const int32_t* row, const int32_t* pos, int32_t n,
                             const ss_rows* k, const ss_rows* v, void* hip_stream)
{
    ss::clear_error();
    if (int rc = check_page_tokens(pages, table, k, v, row, pos, n)) return rc;
    if (int rc = check_apart(k, "k", pages->n_kv_heads, pages->head_dim)) return rc;
    if (int rc = check_apart(v, "v", pages->n_kv_heads, pages->head_dim)) return rc;
    if (n == 0 || table->n_rows == 0 || table->stride == 0) return SS_OK;
    return launch([&] { ss::launch_pages_read(view(pages), view(table), view(k), view(v), k->dtype, row, pos, n, (hipStream_t)hip_stream); });
}

extern "C" int ss_attention_pages_workspace(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t page_slots, int32_t stride, int32_t n,
                                            int32_t max_length, int32_t group, size_t* bytes)
{
    ss::clear_error();
    if (!bytes) return fail(SS_EINVAL, "bytes is NULL");
    if (head_dim != 64 && head_dim != 128) return fail(SS_EINVAL, "head_dim must be 64 or 128");
    if (!is_page_size(page_slots)) return fail(SS_EINVAL, "page_slots must be 16, 32, 64, 128 or 256");
    if (stride < 0 || (int64_t)stride * page_slots > INT_MAX - 1024) return fail(SS_EINVAL, "rows of negative length or of more than 2^31 positions");
    if (int rc = check_page_attention(n_heads, n_kv_heads, page_slots, stride, n, max_length, group)) return rc;
    *bytes = ss::page_space(plan_of_pages(n_heads, n_kv_heads, head_dim, page_slots, stride, n, max_length, group), n, group, n_kv_heads, head_dim, page_slots, stride).bytes;
    return SS_OK;
}

extern "C" int ss_attention_pages(const ss_pages* pages, const ss_page_table* table, const ss_rows* q, const ss_rows* out, int32_t n_heads,
                                  int32_t n, const int32_t* rows, int32_t max_length, int32_t group, float scale, void* workspace,
                                  size_t workspace_bytes, void* hip_stream)
{
    ss::clear_error();
    if (int rc = check_pages_and_table(pages, table)) return rc;
    if (int rc = check_rows(q, "q")) return rc;
    if (int rc = check_rows(out, "out")) return rc;
    if (int rc = check_page_attention(n_heads, pages->n_kv_heads, table->page_slots, table->stride, n, max_length, group)) return rc;
    if (q->dtype != out->dtype) return fail(SS_EINVAL, "q and out differ in type");
    if (pages->dtype != SS_I8 && pages->dtype != q->dtype) return fail(SS_EINVAL, "pages of 16 bits and q must have the same type");
    if (q->rows < n || out->rows < n) return fail(SS_EINVAL, "q or out has fewer than %d rows", n);
    if (!std::isfinite(scale)) return fail(SS_EINVAL, "scale must be finite");
    if (int rc = check_apart(out, "out", n_heads, pages->head_dim)) return rc;
    if (!rows && n > table->n_rows) return fail(SS_EINVAL, "the table has fewer than %d rows", n);
    if (n == 0) return SS_OK;
    const ss::PagePlan p = plan_of_pages(n_heads, pages->n_kv_heads, pages->head_dim, table->page_slots, table->stride, n, max_length, group);
    const ss::PageSpace space = ss::page_space(p, n, group, pages->n_kv_heads, pages->head_dim, table->page_slots, table->stride);
    if (int rc = check_workspace(workspace, workspace_bytes, space.bytes)) return rc;
    ss::PageAttentionArgs a{};
    a.tiles = p.tiles;
    a.row_blocks = p.row_blocks;
    a.parts = p.parts;
    a.at_once = p.at_once;
    a.part = (float*)workspace;
    a.notes = (char*)workspace + space.notes;
    a.item_counts = (int32_t*)((char*)workspace + space.counts);
    a.items = (char*)workspace + space.items;
    a.items_stride = space.items_stride;
    a.p = view(pages);
    a.t = view(table);
    a.q = view(q);
    a.out = view(out);
    a.rows = rows;
    a.scale = scale;
    a.n = n;
    a.group = group;
    a.heads = n_heads;
    return launch([&] { ss::launch_attention_pages(a, q->dtype, (hipStream_t)hip_stream); });
}

extern "C" int ss_pages_workspace(int32_t n_pages, size_t* bytes)
{
    ss::clear_error();
    if (!bytes) return fail(SS_EINVAL, "bytes is NULL");
    if (n_pages < 1 || n_pages > SS_PAGES_MAX) return fail(SS_EINVAL, "there must be a page, and at most %d pages", SS_PAGES_MAX);
    *bytes = pages_workspace(n_pages);
    return SS_OK;
}

extern "C" int ss_pages_fork(const ss_page_table* from, const ss_page_table* to, const int32_t* parent, const int32_t* grow,
                             const uint8_t* held, int32_t* src, int32_t* dst, int32_t* missing, void* workspace, size_t workspace_bytes,
                             void* hip_stream)
{
    ss::clear_error();
    if (int rc = check_two_tables(from, to)) return rc;
    if ((to->n_rows > 0 && (!src || !dst)) || !missing) return fail(SS_EINVAL, "src, dst or missing is NULL");
    if (tables_meet(from, to, false)) return fail(SS_EINVAL, "to must not be from, or share memory with it: rows change places");
    if (int rc = check_workspace(workspace, workspace_bytes, pages_workspace(to->n_pages))) return rc;
    ss::ForkArgs a{view(from), view(to), parent, grow, held, src, dst, missing, (int32_t*)workspace};
    return launch([&] { ss::launch_pages_fork(a, (hipStream_t)hip_stream); });
}

extern "C" int ss_pages_compact(const ss_page_table* from, const ss_page_table* to, const uint8_t* held, int32_t* src, int32_t* dst,
                                int32_t* place, int32_t* counts, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    ss::clear_error();
    if (int rc = check_two_tables(from, to)) return rc;
    if (from->n_rows != to->n_rows || from->stride != to->stride) return fail(SS_EINVAL, "from and to differ in rows or stride");
    if (tables_meet(from, to, true)) return fail(SS_EINVAL, "to must be from itself, or share no memory with it");
    if ((from->n_pages > 1 && (!src || !dst)) || !counts) return fail(SS_EINVAL, "src, dst or counts is NULL");
    if (int rc = check_workspace(workspace, workspace_bytes, pages_workspace(from->n_pages))) return rc;
    ss::CompactArgs a{view(from), view(to), held, src, dst, place, counts, (int32_t*)workspace, (int32_t*)workspace + from->n_pages};
    return launch([&] { ss::launch_pages_compact(a, (hipStream_t)hip_stream); });
}

extern "C" int ss_pages_copy(const ss_pages* layers, int32_t n_layers, const int32_t* src, const int32_t* dst, int32_t n, const int32_t* count,
                             void* hip_stream)
{
    ss::clear_error();
    if (n_layers < 0 || n < 0) return fail(SS_EINVAL, "negative number of layers or pages");
    if (n_layers > 0 && !layers) return fail(SS_EINVAL, "layers is NULL");
    for (int32_t l = 0; l < n_layers; ++l) {
        if (int rc = check_pages(layers + l)) return rc;
        const ss_pages &x = layers[l], &y = layers[0];
        if (x.n_pages != y.n_pages || x.page_slots != y.page_slots || x.n_kv_heads != y.n_kv_heads || x.head_dim != y.head_dim || x.dtype != y.dtype)
            return fail(SS_EINVAL, "layer %d is not like the first", l);
    }
    if (n > 0 && (!src || !dst)) return fail(SS_EINVAL, "src or dst is NULL");
    if (n == 0 || n_layers == 0) return SS_OK;
    std::vector<ss::PagesView> views;
    return ss::no_throw([&] {
        for (int32_t l = 0; l < n_layers; ++l) views.push_back(view(layers + l));
        return launch([&] { ss::launch_pages_copy(views.data(), n_layers, src, dst, n, count, (hipStream_t)hip_stream); });
    });
}

extern "C" int ss_beam_select_workspace(int32_t n_groups, int32_t beams, int32_t vocab, int32_t keep, size_t* bytes)
{
    ss::clear_error();
    if (!bytes) return fail(SS_EINVAL, "bytes is NULL");
    if (int rc = check_beams(n_groups, beams, vocab, keep)) return rc;
    *bytes = beam_workspace(n_groups, beams, vocab, keep);
    return SS_OK;
}

extern "C" int ss_beam_select(const void* logits, int32_t dtype, int64_t row_stride, int32_t n_groups, int32_t beams, int32_t vocab, int32_t keep,
                              const ss_beams* now, const ss_beams* next, int32_t* parent, int32_t* token, int32_t end_id, float length_power,
                              void* workspace, size_t workspace_bytes, void* hip_stream)
{
    ss::clear_error();
    if (int rc = check_beams(n_groups, beams, vocab, keep)) return rc;
    if (dtype != SS_F32 && !is_half(dtype)) return fail(SS_EINVAL, "logits: dtype must be SS_F32, SS_F16 or SS_BF16");
    if (!now || !next) return fail(SS_EINVAL, "now or next is NULL");
    if (end_id < -1 || end_id >= vocab) return fail(SS_EINVAL, "end_id must be -1 or a token");
    if (!std::isfinite(length_power)) return fail(SS_EINVAL, "length_power must be finite");
    if (row_stride < 0 || row_stride > (1ll << 40)) return fail(SS_EINVAL, "logits: row_stride must be 0 to 2^40");
    if ((uintptr_t)logits % (dtype == SS_F32 ? 4 : 2)) return fail(SS_EINVAL, "logits are not aligned as their elements");
    if (!now->history != !next->history) return fail(SS_EINVAL, "now and next both have histories, or neither");
    if (now->history && (now->history_stride < 0 || next->history_stride < 0)) return fail(SS_EINVAL, "negative history_stride");
    if ((length_power != 0.f || now->history || next->lengths) && !now->lengths) return fail(SS_EINVAL, "lengths is NULL: histories, new lengths and length_power need them");
    if (n_groups == 0) return SS_OK;
    if (!logits || !now->totals || !next->totals || !parent || !token) return fail(SS_EINVAL, "logits, totals, parent or token is NULL");
    if (now->totals == next->totals || (now->lengths && now->lengths == next->lengths) || (now->ended && now->ended == next->ended) ||
        (now->history && now->history == next->history))
        return fail(SS_EINVAL, "next must not be now: beams change places");
    if (int rc = check_workspace(workspace, workspace_bytes, beam_workspace(n_groups, beams, vocab, keep))) return rc;
    ss::BeamArgs a{};
    a.logits = logits;
    a.row_stride = row_stride;
    a.n_groups = n_groups;
    a.beams = beams;
    a.vocab = vocab;
    a.keep = keep;
    a.slices = ss::beam_slices(n_groups, beams, vocab, keep, dtype == SS_F32 ? 4 : 2, compute_units());
    a.totals = now->totals;
    a.lengths = now->lengths;
    a.ended = now->ended;
    a.history = now->history;
    a.history_stride = now->history_stride;
    a.next_totals = next->totals;
    a.next_lengths = next->lengths;
    a.next_ended = next->ended;
    a.next_history = next->history;
    a.next_history_stride = next->history_stride;
    a.parent = parent;
    a.token = token;
    a.end_id = end_id;
    a.power = length_power;
    a.part = (float*)workspace;
    return launch([&] { ss::launch_beam_select(a, dtype, (hipStream_t)hip_stream); });
}

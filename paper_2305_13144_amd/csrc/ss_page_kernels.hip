// Kernels of the operators on caches in pages: tokens into and out of their pages, the attention of single tokens over them, the tables
// of rows that fork, grow and end, and the copies that follow from those.
#include "ss_operator_device.h"
#include "ss_plan.h"

#include <climits>

namespace ss {

// ------------------------------------------------------------------------------------------ tables
__device__ __forceinline__ int row_length(const TableView& t, int i) { return min(max(t.lengths[i], 0), t.stride * t.page); }
__device__ __forceinline__ bool is_page(const TableView& t, int p) { return p >= 0 && p < t.n_pages; }
__device__ __forceinline__ int pages_of(int length, int page) { return (length + page - 1) / page; }

// ------------------------------------------------------------------------------------------ write and read
// As k_cache_write: a vector of HD elements is HD / 8 neighbouring lanes', 16 bytes each; a workgroup takes 16 tokens through kPagePasses passes
// over 128 / HD heads, keys and values in different workgroups.
constexpr int kPagePasses = 4, kPageTokens = 16;

// Of a lane: its token, that token's vector of head 0 in the pool (-1: none), its first head.
struct PagePlace {
    int t, head;
    int64_t at;
    static constexpr int step(int hd) { return 128 / hd; }   // heads of a pass
    __device__ __forceinline__ PagePlace(const TableView& tb, int n_kv, const int32_t* row, const int32_t* pos, int n, int vector, int hd)
    {
        t = blockIdx.x * kPageTokens + vector % kPageTokens;
        head = blockIdx.y * (kPagePasses * step(hd)) + vector / kPageTokens;
        at = -1;
        if (t >= n) return;
        const int r = row ? row[t] : t;
        if (r < 0 || r >= tb.rows) return;
        const int len = row_length(tb, r), s = row ? pos[t] : len - 1;
        if (s < 0 || s >= len) return;
        const int p = tb.pages[(int64_t)r * tb.stride + s / tb.page];
        if (is_page(tb, p)) at = (int64_t)p * n_kv * tb.page + s % tb.page;
    }
};

template <int HD, typename TOKEN, typename CACHE>
__global__ __launch_bounds__(256) void k_pages_write(PagesView c, TableView tb, RowsView k, RowsView v, const int32_t* __restrict__ row,
                                                     const int32_t* __restrict__ pos, int n)
{
    constexpr int LPV = HD / 8, STEP = PagePlace::step(HD);
    const bool values = blockIdx.z;
    const RowsView src = values ? v : k;
    const int part = threadIdx.x % LPV;
    const PagePlace at(tb, c.n_kv, row, pos, n, threadIdx.x / LPV, HD);
    u32x4 in[kPagePasses];
    int64_t to[kPagePasses];
#pragma unroll
    for (int p = 0; p < kPagePasses; ++p) {   // beyond the last token or head: read again, written nowhere
        const int h = at.head + p * STEP;
        in[p] = __builtin_nontemporal_load((const u32x4*)((const TOKEN*)src.p + (int64_t)min(at.t, n - 1) * src.row + (int64_t)min(h, c.n_kv - 1) * src.head + part * 8));
        to[p] = at.at >= 0 && h < c.n_kv ? at.at + (int64_t)h * c.page : -1;
    }
#pragma unroll
    for (int p = 0; p < kPagePasses; ++p) {
        if constexpr (std::is_same<CACHE, TOKEN>::value) {
            if (to[p] >= 0) *(u32x4*)((CACHE*)(values ? c.v : c.k) + to[p] * HD + part * 8) = in[p];
        } else {
            float x[8];
            to_floats<TOKEN>(in[p], x);
            if constexpr (std::is_same<CACHE, int8_t>::value) {
                uint2 codes;
                const float scale = quantise<HD>(x, &codes);
                if (to[p] < 0) continue;
                *(uint2*)((int8_t*)(values ? c.v : c.k) + to[p] * HD + part * 8) = codes;
                if (part == 0) (values ? c.v_scale : c.k_scale)[to[p]] = scale;
            } else {
                if (to[p] >= 0) *(u32x4*)((CACHE*)(values ? c.v : c.k) + to[p] * HD + part * 8) = from_floats<CACHE>(x);
            }
        }
    }
}

template <int HD, typename TOKEN, typename CACHE>
__global__ __launch_bounds__(256) void k_pages_read(PagesView c, TableView tb, RowsView k, RowsView v, const int32_t* __restrict__ row,
                                                    const int32_t* __restrict__ pos, int n)
{
    constexpr int LPV = HD / 8, STEP = PagePlace::step(HD);
    const bool values = blockIdx.z;
    const RowsView dst = values ? v : k;
    const int part = threadIdx.x % LPV;
    const PagePlace at(tb, c.n_kv, row, pos, n, threadIdx.x / LPV, HD);
    if (at.at < 0) return;
    u32x4 in[kPagePasses];
    float scale[kPagePasses];
    TOKEN* to[kPagePasses];
#pragma unroll
    for (int p = 0; p < kPagePasses; ++p) {
        const int h = at.head + p * STEP;
        to[p] = nullptr;
        if (h >= c.n_kv) continue;
        const int64_t from = at.at + (int64_t)h * c.page;
        to[p] = (TOKEN*)dst.p + (int64_t)at.t * dst.row + (int64_t)h * dst.head + part * 8;
        const CACHE* src = (const CACHE*)(values ? c.v : c.k) + from * HD + part * 8;
        if constexpr (std::is_same<CACHE, int8_t>::value) {
            const uint2 w = *(const uint2*)src;
            in[p] = u32x4{w.x, w.y, 0u, 0u};
            scale[p] = (values ? c.v_scale : c.k_scale)[from];
        } else {
            in[p] = *(const u32x4*)src;
        }
    }
#pragma unroll
    for (int p = 0; p < kPagePasses; ++p) {
        if (!to[p]) continue;
        if constexpr (std::is_same<CACHE, TOKEN>::value) {
            *(u32x4*)to[p] = in[p];
        } else {
            float x[8];
            if constexpr (std::is_same<CACHE, int8_t>::value) codes_to_floats(make_uint2(in[p][0], in[p][1]), scale[p], x);
            else to_floats<CACHE>(in[p], x);
            __builtin_nontemporal_store(from_floats<TOKEN>(x), (u32x4*)to[p]);
        }
    }
}

// ------------------------------------------------------------------------------------------ attention
// A workgroup takes one query head of one row: a thread a position, then a thread an element.
template <int HD, typename T, typename C>
__global__ __launch_bounds__(256) void k_attention_pages(PageAttentionArgs a)
{
    constexpr bool I8 = std::is_same<C, int8_t>::value;
    __shared__ float s_q[HD], s_p[256], s_red[4];
    __shared__ int64_t s_at[256];
    const int h = blockIdx.x, j = blockIdx.y, hk = h / (a.heads / a.p.n_kv), t = threadIdx.x, P = a.t.page;
    const int r = a.rows ? a.rows[j] : j;
    const int len = r >= 0 && r < a.t.rows ? row_length(a.t, r) : 0;
    if (t < HD) s_q[t] = (float)((const T*)a.q.p)[(int64_t)j * a.q.row + (int64_t)h * a.q.head + t] * a.scale;
    float m = kLowest, l = 0.f, o = 0.f;
    for (int s0 = 0; s0 < len; s0 += 256) {
        __syncthreads();
        const int s = s0 + t;
        int64_t at = -1;
        if (s < len) {
            const int p = a.t.pages[(int64_t)r * a.t.stride + s / P];
            if (is_page(a.t, p)) at = ((int64_t)p * a.p.n_kv + hk) * P + s % P;
        }
        float x = -__builtin_inff();
        if (at >= 0) {
            x = 0.f;
            for (int e = 0; e < HD; ++e) x = fmaf(s_q[e], (float)((const C*)a.p.k)[at * HD + e], x);
            if constexpr (I8) x *= a.p.k_scale[at];
        }
        const float top = wave_max(x);
        if ((t & 63) == 0) s_red[t >> 6] = top;
        __syncthreads();
        const float m_new = fmaxf(m, fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])));
        const float alpha = __expf(m - m_new), p = at >= 0 ? __expf(x - m_new) : 0.f;
        m = m_new;
        __syncthreads();
        const float sum = wave_sum(p);
        if ((t & 63) == 0) s_red[t >> 6] = sum;
        s_p[t] = p;
        s_at[t] = at;
        __syncthreads();
        l = l * alpha + ((s_red[0] + s_red[1]) + (s_red[2] + s_red[3]));
        o *= alpha;
        if (t < HD)
            for (int i = 0; i < 256; ++i)
                if (s_at[i] >= 0) o = fmaf(s_p[i], (float)((const C*)a.p.v)[s_at[i] * HD + t] * (I8 ? a.p.v_scale[s_at[i]] : 1.f), o);
    }
    if (t >= HD) return;
    o = l != 0.f ? o / l : 0.f;
    T* to = (T*)a.out.p + (int64_t)j * a.out.row + (int64_t)h * a.out.head + t;
    if constexpr (std::is_same<T, _Float16>::value) *to = __builtin_bit_cast(_Float16, f2h(o));
    else *to = (T)o;
}

// ------------------------------------------------------------------------------------------ fork
// Three launches.  Claims: of each page the lowest row of `to` that writes into it, -1 if a row holds it that does not (or somebody else
// does), INT_MAX if none does, as one minimum over all entries.  Then every workgroup knows from the claims which pages are free and how many each
// row needs, and the workgroup that has the k-th free page finds the row that gets it.
constexpr int kFree = INT_MAX;

__global__ __launch_bounds__(256) void k_pages_claims(int32_t* __restrict__ claim, const uint8_t* __restrict__ held, int n)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) claim[i] = held && held[i] ? -1 : kFree;
}

// What a row of `to` starts from and becomes.
struct Fork {
    int parent, old_len, new_len, held, wanted, last;   // last: entry of the page that it grows into, or -1
    __device__ __forceinline__ Fork(const ForkArgs& a, int i)
    {
        parent = a.parent ? a.parent[i] : i;
        if (parent < 0 || parent >= a.from.rows) parent = -1;
        const int most = a.to.stride * a.to.page;
        old_len = parent >= 0 ? min(row_length(a.from, parent), most) : 0;
        const int more = a.grow ? max(a.grow[i], 0) : parent >= 0;
        new_len = more < most - old_len ? old_len + more : most;
        held = pages_of(old_len, a.to.page);
        wanted = pages_of(new_len, a.to.page);
        last = new_len > old_len && old_len % a.to.page ? held - 1 : -1;
    }
    __device__ __forceinline__ int page(const ForkArgs& a, int entry) const { return a.from.pages[(int64_t)parent * a.from.stride + entry]; }
    // The page that row i must not write into, or -1.
    __device__ __forceinline__ int shared(const ForkArgs& a, int i) const
    {
        if (last < 0) return -1;
        const int p = page(a, last);
        return is_page(a.from, p) && a.claim[p] != i ? p : -1;
    }
};

__global__ __launch_bounds__(256) void k_pages_inherit(ForkArgs a)
{
    const int i = blockIdx.x;
    const Fork f(a, i);
    for (int k = threadIdx.x; k < a.to.stride; k += 256) {
        int p = -1;
        if (k < f.held) {
            p = f.page(a, k);
            if (!is_page(a.from, p)) p = -1;
            else atomicMin(&a.claim[p], k == f.last ? i : -1);
        }
        a.to.pages[(int64_t)i * a.to.stride + k] = p;
    }
    if (threadIdx.x == 0) {
        a.to.lengths[i] = f.new_len;
        a.src[i] = a.dst[i] = -1;
    }
}

// Sum over the workgroup's NT threads, in each of them, and of those before a thread.
template <int NT>
struct Scan {
    int before, all;
    __device__ __forceinline__ Scan(int x, int* lds)   // lds: NT / 64 + 1
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        int s = x;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(s, d);
            if (lane >= d) s += o;
        }
        __syncthreads();
        if (lane == 63) lds[wave] = s;
        __syncthreads();
        before = s - x;
        all = 0;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) {
            if (w < wave) before += lds[w];
            all += lds[w];
        }
    }
};

constexpr int kForkThreads = 1024, kForkPages = 4096;   // pages of a workgroup

__global__ __launch_bounds__(kForkThreads) void k_pages_hand_out(ForkArgs a)
{
    extern __shared__ int s_start[];   // [rows + 1] first of each row's pages among those handed out
    __shared__ int s_scan[kForkThreads / 64 + 1];
    const int rows = a.to.rows, n = a.to.n_pages, t = threadIdx.x, first = blockIdx.x * kForkPages;
    int total = 0;
    for (int r0 = 0; r0 < rows; r0 += kForkThreads) {
        const int i = r0 + t;
        int need = 0;
        if (i < rows) {
            const Fork f(a, i);
            need = f.wanted - f.held + (f.shared(a, i) >= 0);
        }
        const Scan<kForkThreads> s(need, s_scan);
        if (i < rows) s_start[i] = total + s.before;
        total += s.all;
    }
    int mine = 0, ahead = 0, every = 0;   // free pages of this thread (4 neighbours), before this workgroup, at all
    for (int p0 = 0; p0 < n; p0 += kForkPages) {
        int free_here = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int p = p0 + 4 * t + k;
            free_here += p < n && a.claim[p] == kFree;
        }
        if (p0 == first) mine = free_here;
        if (p0 < first) ahead += free_here;
        every += free_here;
    }
    every = Scan<kForkThreads>(every, s_scan).all;
    ahead = Scan<kForkThreads>(ahead, s_scan).all;
    int rank = ahead + Scan<kForkThreads>(mine, s_scan).before;
    __syncthreads();
    auto give = [&](int rank, int page) {   // the rank-th page that is needed
        int lo = 0, hi = rows - 1;          // the last row whose first is not behind it
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (s_start[mid] <= rank) lo = mid;
            else hi = mid - 1;
        }
        const Fork f(a, lo);
        const int shared = f.shared(a, lo), k = rank - s_start[lo] - (shared >= 0);
        a.to.pages[(int64_t)lo * a.to.stride + (k < 0 ? f.last : f.held + k)] = page;
        if (k < 0 && page >= 0) {
            a.src[lo] = shared;
            a.dst[lo] = page;
        }
    };
    for (int k = 0; k < 4; ++k) {
        const int p = first + 4 * t + k;
        if (p < n && a.claim[p] == kFree && rank < total) give(rank++, p);
    }
    if (blockIdx.x > 0) return;
    for (int k = every + t; k < total; k += kForkThreads) give(k, -1);
    if (t == 0) *a.missing = max(total - every, 0);
}

// ------------------------------------------------------------------------------------------ compact
__global__ __launch_bounds__(256) void k_pages_unused(int32_t* __restrict__ used, const uint8_t* __restrict__ held, int n)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) used[i] = held && held[i];
}

__global__ __launch_bounds__(256) void k_pages_mark(CompactArgs a)
{
    const int i = blockIdx.x, n = pages_of(row_length(a.from, i), a.from.page);
    for (int k = threadIdx.x; k < n; k += 256) {
        const int p = a.from.pages[(int64_t)i * a.from.stride + k];
        if (is_page(a.from, p)) a.used[p] = 1;
    }
}

// code: a page's new number, -1 if it is free, -2 - k if it is the k-th that moves.
__global__ __launch_bounds__(kForkThreads) void k_pages_rank(CompactArgs a)
{
    __shared__ int s_scan[kForkThreads / 64 + 1];
    const int n = a.from.n_pages, t = threadIdx.x, first = blockIdx.x * kForkPages;
    int mine = 0, ahead = 0, every = 0, below = 0;
    for (int p0 = 0; p0 < n; p0 += kForkPages) {
        int here = 0;
        for (int k = 0; k < 4; ++k) {
            const int p = p0 + 4 * t + k;
            here += p < n && a.used[p];
        }
        if (p0 == first) mine = here;
        if (p0 < first) ahead += here;
        every += here;
    }
    every = Scan<kForkThreads>(every, s_scan).all;
    ahead = Scan<kForkThreads>(ahead, s_scan).all;
    for (int p = t; p < every; p += kForkThreads) below += a.used[p] != 0;
    below = Scan<kForkThreads>(below, s_scan).all;      // pages in use that keep their numbers
    const int moves = every - below;
    int used_before = ahead + Scan<kForkThreads>(mine, s_scan).before;
    for (int k = 0; k < 4; ++k) {
        const int p = first + 4 * t + k;
        if (p >= n) break;
        const bool used = a.used[p];
        int code = used ? p : -1;
        if (used && p >= every) {
            const int rank = used_before - below;
            a.src[rank] = p;
            code = -2 - rank;
        } else if (!used && p < every) {
            a.dst[p - used_before] = p;
        }
        a.code[p] = code;
        if (p >= moves && p < n / 2) a.src[p] = a.dst[p] = -1;
        used_before += used;
    }
    if (blockIdx.x == 0 && t == 0) {
        a.counts[0] = every;
        a.counts[1] = moves;
    }
}

__global__ __launch_bounds__(256) void k_pages_renumber(CompactArgs a)
{
    auto place = [&](int p) {
        const int code = a.code[p];
        return code <= -2 ? a.dst[-2 - code] : code;
    };
    if ((int)blockIdx.x >= a.from.rows) {
        const int p = (blockIdx.x - a.from.rows) * 256 + threadIdx.x;
        if (a.place && p < a.from.n_pages) a.place[p] = place(p);
        return;
    }
    const int i = blockIdx.x, len = row_length(a.from, i), n = pages_of(len, a.from.page);
    for (int k = threadIdx.x; k < a.from.stride; k += 256) {
        const int64_t at = (int64_t)i * a.from.stride + k;
        const int p = k < n ? a.from.pages[at] : -1;
        a.to.pages[at] = is_page(a.from, p) ? place(p) : -1;
    }
    if (threadIdx.x == 0) a.to.lengths[i] = len;
}

// ------------------------------------------------------------------------------------------ copies
constexpr int kCopyLayers = 32;   // of a launch
struct CopyArgs {
    void* p[kCopyLayers][2];
    float* scale[kCopyLayers][2];
    const int32_t *src, *dst, *count;
    int n, n_pages;
    int64_t bytes, scale_bytes;   // of a page
};

__global__ __launch_bounds__(256) void k_pages_copy(CopyArgs a)
{
    const int layer = blockIdx.y >> 1, which = blockIdx.y & 1;
    const int n = a.count ? min(a.n, *a.count) : a.n;
    for (int i = blockIdx.x; i < n; i += gridDim.x) {
        const int s = a.src[i], d = a.dst[i];
        if (s < 0 || s >= a.n_pages || d < 0 || d >= a.n_pages || s == d) continue;
        const char* from = (const char*)a.p[layer][which] + s * a.bytes;
        char* to = (char*)a.p[layer][which] + d * a.bytes;
        for (int64_t k = threadIdx.x * 16; k < a.bytes; k += 256 * 16) *(u32x4*)(to + k) = *(const u32x4*)(from + k);
        if (!a.scale_bytes) continue;
        from = (const char*)a.scale[layer][which] + s * a.scale_bytes;
        to = (char*)a.scale[layer][which] + d * a.scale_bytes;
        for (int64_t k = threadIdx.x * 16; k < a.scale_bytes; k += 256 * 16) *(u32x4*)(to + k) = *(const u32x4*)(from + k);
    }
}

// ------------------------------------------------------------------------------------------ launches
void launch_pages_write(const PagesView& p, const TableView& t, const RowsView& k, const RowsView& v, int token, const int32_t* row,
                        const int32_t* pos, int n, hipStream_t s)
{
    with_types(p.hd, token, p.dtype, [&](auto dim, auto tt, auto e) {
        constexpr int HD = decltype(dim)::value, heads = kPagePasses * PagePlace::step(HD);
        k_pages_write<HD, decltype(tt), decltype(e)><<<dim3((n + kPageTokens - 1) / kPageTokens, (p.n_kv + heads - 1) / heads, 2), 256, 0, s>>>(p, t, k, v, row, pos, n);
    });
}

void launch_pages_read(const PagesView& p, const TableView& t, const RowsView& k, const RowsView& v, int token, const int32_t* row,
                       const int32_t* pos, int n, hipStream_t s)
{
    with_types(p.hd, token, p.dtype, [&](auto dim, auto tt, auto e) {
        constexpr int HD = decltype(dim)::value, heads = kPagePasses * PagePlace::step(HD);
        k_pages_read<HD, decltype(tt), decltype(e)><<<dim3((n + kPageTokens - 1) / kPageTokens, (p.n_kv + heads - 1) / heads, 2), 256, 0, s>>>(p, t, k, v, row, pos, n);
    });
}

void launch_attention_pages(const PageAttentionArgs& a, int token, hipStream_t s)
{
    with_types(a.p.hd, token, a.p.dtype, [&](auto dim, auto t, auto e) {
        typedef decltype(t) T;
        typedef decltype(e) C;
        if constexpr (std::is_same<C, int8_t>::value || std::is_same<C, T>::value)
            k_attention_pages<decltype(dim)::value, T, C><<<dim3(a.heads, a.n), 256, 0, s>>>(a);
    });
}

void launch_pages_fork(const ForkArgs& a, hipStream_t s)
{
    const int n = a.to.n_pages;
    k_pages_claims<<<(n + 255) / 256, 256, 0, s>>>(a.claim, a.held, n);
    k_pages_inherit<<<a.to.rows, 256, 0, s>>>(a);
    k_pages_hand_out<<<(n + kForkPages - 1) / kForkPages, kForkThreads, (size_t)(a.to.rows + 1) * 4, s>>>(a);
}

void launch_pages_compact(const CompactArgs& a, hipStream_t s)
{
    const int n = a.from.n_pages;
    k_pages_unused<<<(n + 255) / 256, 256, 0, s>>>(a.used, a.held, n);
    if (a.from.rows > 0) k_pages_mark<<<a.from.rows, 256, 0, s>>>(a);
    k_pages_rank<<<(n + kForkPages - 1) / kForkPages, kForkThreads, 0, s>>>(a);
    k_pages_renumber<<<a.from.rows + (a.place ? (n + 255) / 256 : 0), 256, 0, s>>>(a);
}

void launch_pages_copy(const PagesView* layers, int n_layers, const int32_t* src, const int32_t* dst, int n, const int32_t* count, hipStream_t s)
{
    for (int first = 0; first < n_layers; first += kCopyLayers) {
        CopyArgs a{};
        const int here = n_layers - first < kCopyLayers ? n_layers - first : kCopyLayers;
        const PagesView& p = layers[first];
        const int64_t vectors = (int64_t)p.n_kv * p.page;
        a.bytes = vectors * p.hd * (p.dtype == kI8 ? 1 : 2);
        a.scale_bytes = p.dtype == kI8 ? vectors * 4 : 0;
        for (int l = 0; l < here; ++l) {
            a.p[l][0] = layers[first + l].k;
            a.p[l][1] = layers[first + l].v;
            a.scale[l][0] = layers[first + l].k_scale;
            a.scale[l][1] = layers[first + l].v_scale;
        }
        a.src = src;
        a.dst = dst;
        a.count = count;
        a.n = n;
        a.n_pages = p.n_pages;
        k_pages_copy<<<dim3(n < 2048 ? n : 2048, 2 * here), 256, 0, s>>>(a);
    }
}

}  // namespace ss

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
// over 128 / HD heads, keys and values in different workgroups.  Bound by the bytes (8746 tokens of 32 heads of 128, halves into 8 bits, written and read:
// 82 us, 4.7 TB/s), a step of few tokens by its chain of loads: row, length and entry come before the slot.
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

// ------------------------------------------------------------------------------------------ attention
// A unit is one key/value head of a group of rows: its rows r = row of the group * G + (head within its G), in blocks of 16 * QT.  Its slots come in
// items: 16 neighbouring slots of one page, with the positions that they are and the rows of the group that hold the page there.  Of a single row the
// items are its table; of a group k_page_items lists every page once per entry, however many rows hold it.
// The mathematics of a step of two items is that of k_attention_tree (ss_cache_kernels.h): S^T = K Q^T, an online softmax in powers of two whose weights
// are the operand of O^T += V^T P^T as they lie, nothing staged in LDS; what differs is where slots lie and who sees them.  An item is always
// whole in memory, so nothing is clamped; scores of slots that a row does not see are set to -inf.  Values of such slots meet weights of 0: in 8 bits
// they are finite whatever lies there (the scale is left out); in 16 bits an infinity or NaN shows in a wave's sums, and the wave goes through its items again with
// such values counting as 0 in steps that not every row sees in all slots (16 x 8 beams with NaN wherever no row looks 66 us, with numbers 48).  Those that some
// row sees are added to its sums at the end, so a row's bits do not depend on what it does not see.
// What is rounded: the weights, to the operand's type.  In 16 bits their sum is of the rounded ones (half 0.00024 of a call, 0.00021 of it the result's own rounding; bf16
// 0.0019 and 0.0016; sums of two would take registers that there are not).  Over 8 bits with results in half they are sums of two halves: 0.00021 instead of
// 0.00029, for a second product beside each (16 x 8 beams 38.0 us, 35.6).
// Bound by the cache's bytes (64 rows to 8000 slots, 32 heads on 8, 8 bits: 439 MB in 88 us with the join, 6.5 TB/s while large parts run, 5.0 in all), with few
// or short rows by a chain of latencies (one row of 3900 slots and 32 heads: 12 us, and 3 of the join).  3 workgroups on a unit (QT == 1, heads of 128): a
// fourth wave a SIMD spills.
// Who takes what (page_plan): short rows a workgroup a unit; one long row, or few that are not very long, a workgroup one of `parts` equal parts of a unit; else
// (DEALT) units are cut by the rows' lengths (PageCuts).  k_page_join adds up the parts of units.
struct PageItem {
    int page, p0;
    unsigned mask;   // rows of the group
    int full;        // seen by all rows of the group in all slots
};
static_assert(sizeof(PageItem) == 16, "four words");

// Of the j-th group: items, and the i-th of them.
__device__ __forceinline__ int attended_row(const PageAttentionArgs& a, int q) { return a.rows ? a.rows[q] : q; }
__device__ __forceinline__ int attended_length(const PageAttentionArgs& a, int r) { return r >= 0 && r < a.t.rows ? row_length(a.t, r) : 0; }
__device__ __forceinline__ int group_items(const PageAttentionArgs& a, int j)
{
    return a.group == 1 ? (attended_length(a, attended_row(a, j)) + 15) >> 4 : a.item_counts[j];
}
__device__ __forceinline__ PageItem group_item(const PageAttentionArgs& a, int j, int row, int len, int i)
{
    if (a.group > 1) return ((const PageItem*)a.items)[(int64_t)j * a.items_stride + i];
    const int p0 = 16 * i, p = a.t.pages[(int64_t)row * a.t.stride + p0 / a.t.page];
    if (!is_page(a.t, p)) return {0, p0, 0u, 0};
    return {p, p0, 1u, p0 + 16 <= len};
}

// The items of a group, by position and there by the first row that holds the page: a round of as many positions as the threads hold, compared through LDS.
// 8 rows of 206 entries: 6.4 us, two rounds of latencies; rows in neighbouring lanes that compare by shuffles, twice through to count first: 7.4.
constexpr int kItemThreads = 1024;
__global__ __launch_bounds__(kItemThreads) void k_page_items(PageAttentionArgs a)
{
    __shared__ int s_page[kItemThreads], s_len[32], s_row[32], s_scan[kItemThreads / 64 + 1];
    const int j = blockIdx.x, g = a.group, t = threadIdx.x, P = a.t.page;
    if (t < g) {
        const int r = attended_row(a, j * g + t);
        s_row[t] = r;
        s_len[t] = attended_length(a, r);
    }
    __syncthreads();
    int most = 0, least = INT_MAX;
    for (int b = 0; b < g; ++b) {
        most = max(most, s_len[b]);
        least = min(least, s_len[b]);
    }
    const int entries = pages_of(most, P), per = kItemThreads / g, b = t % g;
    PageItem* out = (PageItem*)a.items + (int64_t)j * a.items_stride;
    const unsigned all = g == 32 ? ~0u : (1u << g) - 1;
    int count = 0;
    for (int e0 = 0; e0 < entries; e0 += per) {
        const int e = e0 + t / g;
        int page = -1;
        if (t < per * g && e < pages_of(s_len[b], P)) {
            page = a.t.pages[(int64_t)s_row[b] * a.t.stride + e];
            if (!is_page(a.t, page)) page = -1;
        }
        __syncthreads();
        s_page[t] = page;
        __syncthreads();
        unsigned mask = 0;
        int len = 0;
        if (page >= 0)
            for (int c = 0; c < g; ++c)
                if (s_page[t - b + c] == page) {
                    mask |= 1u << c;
                    len = max(len, s_len[c]);
                }
        const int tiles = page >= 0 && __ffs(mask) - 1 == b ? (min(len - e * P, P) + 15) >> 4 : 0;
        const Scan<kItemThreads> s(tiles, s_scan);
        for (int i = 0; i < tiles; ++i) {
            const int p0 = e * P + 16 * i;
            out[count + s.before + i] = {page, p0, mask, mask == all && p0 + 16 <= least};
        }
        count += s.all;
    }
    if (t == 0) a.item_counts[j] = count;
}

template <typename T, int N>
__device__ __forceinline__ void page_store(const PageAttentionArgs& a, int q, int head, int e0, const float (&x)[N])
{
    T r[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (std::is_same<T, _Float16>::value) r[i] = __builtin_bit_cast(_Float16, f2h(x[i]));
        else r[i] = (T)x[i];
    }
    typedef uint32_t words __attribute__((ext_vector_type(N * 2 / 4)));
    *(words*)((T*)a.out.p + (int64_t)q * a.out.row + (int64_t)head * a.out.head + e0) = __builtin_bit_cast(words, r);
}

// What all lanes hold alike, in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)uniform((int)x) | (uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32);
}

__device__ __forceinline__ int64_t lane_value(int64_t x, int l)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)x, l) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32);
}

// Sum over the lanes up to each (DPP controls: rows shifted by 1, 2, 4 and 8, then row ends to the rows behind).
template <int C, int R>
__device__ __forceinline__ int from_before(int x) { return __builtin_amdgcn_update_dpp(0, x, C, R, 0xf, false); }
template <int C, int R>
__device__ __forceinline__ int64_t from_before(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)from_before<C, R>((int)x) | (uint64_t)(uint32_t)from_before<C, R>((int)(x >> 32)) << 32);
}
template <typename I>
__device__ __forceinline__ I wave_prefix(I x)
{
    x += from_before<0x111, 0xf>(x);
    x += from_before<0x112, 0xf>(x);
    x += from_before<0x114, 0xf>(x);
    x += from_before<0x118, 0xf>(x);
    x += from_before<0x142, 0xa>(x);
    x += from_before<0x143, 0xc>(x);
    return x;
}

// The largest number of a row of 16 lanes, in all of them.
__device__ __forceinline__ int row_max(int x)
{
    x = max(x, __builtin_amdgcn_mov_dpp(x, kDppXor1, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_mov_dpp(x, kDppXor2, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_mov_dpp(x, kDppHalfMirror, 0xf, 0xf, false));
    return max(x, __builtin_amdgcn_mov_dpp(x, kDppMirror, 0xf, 0xf, false));
}

// What a workgroup gets: the k-th part of unit hb of group j (j < 0: nothing).  Every wave finds its place by itself, a lane a group (or some), so
// that there is nothing to wait for.
struct PageShare {
    int j, hb, k, count;
    PageCuts cuts;
};
__device__ __forceinline__ PageShare page_share(const PageAttentionArgs& a, int units, int n_groups)
{
    const int lane = threadIdx.x & 63, per = (n_groups + 63) / 64, g0 = min(lane * per, n_groups), g1 = min(g0 + per, n_groups);
    const int only = per == 1 && g0 < g1 ? group_items(a, g0) : 0;
    auto items_of = [&](int j) { return per == 1 ? only : group_items(a, j); };   // of a lane's own group
    int64_t sum = 0;
    for (int j = g0; j < g1; ++j) sum += items_of(j);
    const int64_t all = lane_value(wave_prefix(sum), 63) * units;
    // (a division of 64 bits takes microseconds)
    const int64_t average64 = all < 1 << 30 ? ((uint32_t)all + (uint32_t)a.at_once - 1) / (uint32_t)a.at_once : (all + a.at_once - 1) / a.at_once;
    const int average = uniform((int)min(max(average64, (int64_t)kPageShare), (int64_t)1 << 28));
    PageShare s{-1, 0, 0, 0, {0, average}};
    if (average >= kPageMany) {
        s.cuts = page_large_cuts(average);
    } else {   // three widths at a time; with the widest there is a place for every part, as a unit has one that is not whole
        const int all_units = n_groups * units, places = all_units < a.at_once / 4 * 3 ? a.at_once - all_units : a.at_once;
        const int w2 = uniform((int)(((uint32_t)all + (uint32_t)places - 1) / (uint32_t)places)), w1 = (average + w2) / 2;   // all < 64 * at_once
        int n0 = 0, n1 = 0;
        for (int j = g0; j < g1; ++j) {
            const int n = items_of(j);
            n0 += (int)((uint32_t)(n + average - 1) / (uint32_t)average);
            n1 += (int)((uint32_t)(n + w1 - 1) / (uint32_t)w1);
        }
        auto fits = [&](int n) { return (int64_t)__builtin_amdgcn_readlane(wave_prefix(n), 63) * units <= a.at_once; };
        if (!fits(n0)) s.cuts.small = fits(n1) ? w1 : max(w2, average);
    }
    // all large parts in a row, then all small ones
    int large, small, large_upto, small_upto;   // of a lane's groups, a unit of each
    int64_t all_large;
    auto count_parts = [&] {
        large = small = 0;
        for (int j = g0; j < g1; ++j) {
            const int n = items_of(j);
            large += s.cuts.large_of(n);
            small += s.cuts.small_of(n);
        }
        large_upto = wave_prefix(large);
        small_upto = wave_prefix(small);
        all_large = (int64_t)__builtin_amdgcn_readlane(large_upto, 63) * units;
        return all_large + (int64_t)__builtin_amdgcn_readlane(small_upto, 63) * units;
    };
    if (count_parts() > gridDim.x) {
        s.cuts = page_least_cuts(average, a.group);
        count_parts();
    }
    const bool is_large = (int)blockIdx.x < all_large;
    const int64_t from = is_large ? (int64_t)(large_upto - large) * units : all_large + (int64_t)(small_upto - small) * units;
    int64_t off64 = (int)blockIdx.x - from;
    const bool here = off64 >= 0 && off64 < (int64_t)(is_large ? large : small) * units;
    const uint64_t whose = __ballot(here);
    if (!whose) return s;
    int my_j = g0, my_n = 0, off = (int)off64, parts = 0;
    if (here)
        while (true) {
            my_n = items_of(my_j);
            parts = is_large ? s.cuts.large_of(my_n) : s.cuts.small_of(my_n);
            if (off < parts * units) break;
            off -= parts * units;
            ++my_j;
        }
    const int owner = __ffsll((unsigned long long)whose) - 1;
    s.j = __builtin_amdgcn_readlane(my_j, owner);
    s.count = __builtin_amdgcn_readlane(my_n, owner);
    parts = __builtin_amdgcn_readlane(parts, owner);
    off = __builtin_amdgcn_readlane(off, owner);
    s.hb = uniform((int)((uint32_t)off / (uint32_t)parts));
    s.k = off - s.hb * parts;
    if (!is_large) s.k += uniform(s.cuts.large_of(s.count));
    return s;
}

// Notes for the join: how units are cut, then the first large and the first small part of each unit.
struct PageNotes {
    PageCuts cuts;
    int pad[2];
    int2 first[1];
};

template <int HD, typename T, typename C, int QT, bool DEALT>
__global__ __launch_bounds__(256, QT == 1 ? HD == 64 ? 4 : 3 : 2) void k_attention_pages(PageAttentionArgs a)
{
    typedef typename MathType<C, T>::type M;
    typedef typename Half<M>::x8 m8;
    constexpr bool I8 = std::is_same<C, int8_t>::value;
    constexpr int KS = HD / 32, ET = HD / 16, NW = 4, ROWS = 16 * QT;
    constexpr int ROW = HD * sizeof(C);      // bytes of a vector
    constexpr int KL = ROW / 64;             // 16-byte loads per 16 slots and lane
    constexpr int VW = ET * sizeof(C) / 4;   // words per slot and lane: ET elements
    constexpr bool PAIRS = I8 && std::is_same<T, _Float16>::value;   // weights as sums of two halves: bf16 results round off more than one leaves
    __shared__ float s_m[NW][ROWS], s_l[NW][ROWS];
    __shared__ int s_odd[NW];
    __shared__ __attribute__((aligned(16))) float s_o[NW][QT][4][64][ET];

    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), ql = lane & 15, g = lane >> 4;
    const int n_kv = a.p.n_kv, G = a.heads / n_kv, units = n_kv * a.row_blocks, n_groups = a.n / a.group, P = a.t.page;
    const int unit_rows = a.group * G;

    // ---- one unit's items i0 .. i1 - 1, all of them if whole; else the sums go to part
    auto piece = [&](int j, int hb, int i0, int i1, bool whole, float* part) {
        const int rb = hb / n_kv, h = hb - rb * n_kv, r0 = rb * ROWS, n_rows = min(unit_rows - r0, ROWS);
        const int row0 = uniform(attended_row(a, j * a.group)), len0 = a.group == 1 ? uniform(attended_length(a, row0)) : 0;
        const char *K = (const char*)a.p.k + (int64_t)h * P * ROW, *V = (const char*)a.p.v + (int64_t)h * P * ROW;
        const float *kscale = I8 ? a.p.k_scale + (int64_t)h * P : nullptr, *vscale = I8 ? a.p.v_scale + (int64_t)h * P : nullptr;

        // A step's operands as they come from memory; those of the next step are requested as soon as the registers are free.
        u32x4 kreg[2][KL];
        uint32_t vreg[8][VW];
        f32x4 ks[2], vs[2];
        const unsigned k_off = ql * ROW + 16 * g, v_off = 4 * g * ROW + ET * ql * (int)sizeof(C);
        auto load16 = [](const char* p) { return __builtin_nontemporal_load((const u32x4*)p); };
        auto slot_of = [&](int page, int p0) { return (int64_t)page * ((int64_t)n_kv * P) + (p0 & (P - 1)); };   // of head 0
        auto load_keys = [&](const int64_t (&at)[2]) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const char* p = K + at[kt] * ROW;
#pragma unroll
                for (int i = 0; i < KL; ++i) kreg[kt][i] = load16(p + k_off + 64 * i);
                if constexpr (I8) ks[kt] = *(const f32x4*)(kscale + at[kt] + 4 * g);
            }
        };
        auto load_values = [&](const int64_t (&at)[2]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const char* p = V + at[i >> 2] * ROW + v_off + (i & 3) * ROW;
                if constexpr (VW == 4) {
                    const u32x4 w = load16(p);
#pragma unroll
                    for (int e = 0; e < 4; ++e) vreg[i][e] = w[e];
                } else if constexpr (VW == 2) {
                    const u32x2 w = __builtin_nontemporal_load((const u32x2*)p);
                    vreg[i][0] = w[0];
                    vreg[i][1] = w[1];
                } else {
                    vreg[i][0] = __builtin_nontemporal_load((const uint32_t*)p);
                }
            }
            if constexpr (I8)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) vs[kt] = *(const f32x4*)(vscale + at[kt] + 4 * g);
        };

        // queries, and what brings their scores to units of log2, as in k_attention_tree
        constexpr bool SCALED = !I8 || !std::is_same<M, T>::value;   // sc is not 1
        const float log2_scale = a.scale * 1.44269504088896341f;
        float sc[QT];
        m8 qf[QT][KS];
        int len[QT], bit[QT];   // of this lane's row: its length and its place in the group
        u32x4 qreg[QT][KS];
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            const int r = min(r0 + u * 16 + ql, unit_rows - 1), b = r / G;
            const T* qp = (const T*)a.q.p + (int64_t)(j * a.group + b) * a.q.row + (int64_t)(h * G + r - b * G) * a.q.head;
#pragma unroll
            for (int i = 0; i < KS; ++i) qreg[u][i] = *(const u32x4*)(I8 ? qp + 64 * (i >> 1) + 16 * g + 8 * (i & 1) : qp + 32 * i + 8 * g);
            bit[u] = b;
            len[u] = a.group == 1 ? len0 : attended_length(a, attended_row(a, j * a.group + b));
        }
        f32x4 o[QT][ET];
        float m_run[QT], l_run[QT];
        WeightUnit unit[QT];
        bool odd = false;
        // A wave takes every fourth step of two items; its lanes hold those of its next 32 steps.
        const int n_items = i1 - i0, steps = (n_items + 1) >> 1;
        PageItem held;
        auto fetch = [&](int step) {
            const int i = 2 * (step + NW * (lane >> 1)) + (lane & 1);
            held = PageItem{0, 0, 0u, 0};
            if (i < n_items) held = group_item(a, j, row0, len0, i0 + i);
        };
        int p0[2], full = 0, turn = 0;   // of the step whose operands are under way
        unsigned mask[2];
        int64_t at[2];
        auto place = [&](int step) {
            if ((turn & 31) == 0) fetch(step);
            full = 1;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const int l = 2 * (turn & 31) + kt;
                p0[kt] = __builtin_amdgcn_readlane(held.p0, l);
                mask[kt] = (unsigned)__builtin_amdgcn_readlane((int)held.mask, l);
                full &= __builtin_amdgcn_readlane(held.full, l);
                at[kt] = slot_of(__builtin_amdgcn_readlane(held.page, l), p0[kt]);
            }
            ++turn;
        };
#pragma unroll
        for (int pass = 0; pass < (I8 ? 1 : 2); ++pass) {
            const bool again = pass > 0;   // (nothing is requested ahead then: there are no registers for it)
            turn = 0;
#pragma unroll
            for (int u = 0; u < QT; ++u) {
#pragma unroll
                for (int e = 0; e < ET; ++e) o[u][e] = (f32x4){0.f, 0.f, 0.f, 0.f};
                m_run[u] = kLowest;
                l_run[u] = 0.f;
            }
            if (wave < steps) {
                place(wave);
                load_keys(at);
                load_values(at);
            }
            // made into operands here, behind the first requests: sooner, those would wait for the queries (one row of 3900 slots in 16 bits 17.0 us, 17.3)
            if constexpr (std::is_same<M, T>::value) {
                const uint32_t flip = !I8 && a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
                for (int u = 0; u < QT; ++u) {
                    sc[u] = I8 ? 1.f : fmaxf(fabsf(log2_scale), 1e-37f);
#pragma unroll
                    for (int i = 0; i < KS; ++i) qf[u][i] = __builtin_bit_cast(m8, qreg[u][i] ^ u32x4{flip, flip, flip, flip});
                }
            } else {   // bf16 queries, half arithmetic: the largest magnitude of each row becomes 2^14 to 2^15
#pragma unroll
                for (int u = 0; u < QT; ++u) {
                    float top = 0.f, x[8];
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        to_floats<T>(qreg[u][i], x);
#pragma unroll
                        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
                    }
                    top = across<32>(across<16>(top, Max()), Max());
                    const float down = half_power(top, &sc[u]);
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        to_floats<T>(qreg[u][i], x);
#pragma unroll
                        for (int e = 0; e < 8; ++e) qf[u][i][e] = (_Float16)(x[e] * down);
                    }
                }
            }
            for (int step = wave; step < steps; step += NW) {
                const bool more = step + NW < steps;
                const int it_p0[2] = {p0[0], p0[1]}, all = full;
                const unsigned it_mask[2] = {mask[0], mask[1]};
                if (more) place(step + NW);
                f32x4 s[QT][2];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    m8 kf[KS];
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        if constexpr (I8) {
                            const uint32_t lo = kreg[kt][i >> 1][2 * (i & 1)], up = kreg[kt][i >> 1][2 * (i & 1) + 1];
                            const u32x4 w = {code_pair(lo, lo, 0x0c010c00u), code_pair(lo, lo, 0x0c030c02u), code_pair(up, up, 0x0c010c00u),
                                             code_pair(up, up, 0x0c030c02u)};
                            kf[i] = __builtin_bit_cast(m8, w);
                        } else {
                            kf[i] = __builtin_bit_cast(m8, kreg[kt][i]);
                        }
                    }
#pragma unroll
                    for (int u = 0; u < QT; ++u) {
                        s[u][kt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int i = 0; i < KS; ++i) s[u][kt] = Half<M>::mma(kf[i], qf[u][i], s[u][kt]);
                    }
                }
                f32x4 kq[2];
                if constexpr (I8)
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) kq[kt][i] = ks[kt][i] * log2_scale;
                if (!again && more) load_keys(at);
                m8 pb[QT], rest[QT];
#pragma unroll
                for (int u = 0; u < QT; ++u) {
                    f32x4 w[2];   // the values' scales, 0 for those that the row does not see
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt) {
                        if constexpr (I8) {
                            w[kt] = vs[kt];
#pragma unroll
                            for (int i = 0; i < 4; ++i) s[u][kt][i] *= kq[kt][i];
                        }
                        if (!all) {
                            const int seen = it_mask[kt] >> bit[u] & 1 ? len[u] - it_p0[kt] - 4 * g : 0;   // of this lane's four slots
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (i >= seen) {
                                    s[u][kt][i] = -__builtin_inff();
                                    if constexpr (I8) w[kt][i] = 0.f;
                                }
                        }
                    }
                    float mt = kLowest;
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) mt = fmaxf(mt, s[u][kt][i]);
                    mt = across<32>(across<16>(mt, Max()), Max());
                    // the weights are relative to a maximum that is followed in steps of 2^8: half holds 2^8 as well as 1; each row's by itself, as all that follows
                    float alpha = 1.f;
                    const bool moves = (mt - m_run[u]) * sc[u] > 8.f, any_moves = __any(moves);
                    if (any_moves) {
                        const float m_new = moves ? mt : m_run[u];
                        alpha = __builtin_amdgcn_exp2f((m_run[u] - m_new) * sc[u]);
                        m_run[u] = m_new;
                        l_run[u] *= alpha;
                        if constexpr (!I8)
#pragma unroll
                            for (int e = 0; e < ET; ++e) o[u][e] *= alpha;
                    }
                    const float m_sc = I8 ? fmaxf(m_run[u] * sc[u], kLowest) : exponent_top<true>(m_run[u], sc[u], s[u]);   // 8 bits: sc is a power of two
                    float top = 0.f;
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float p = __builtin_amdgcn_exp2f(SCALED ? fmaf(s[u][kt][i], sc[u], -m_sc) : below_top(s[u][kt][i], m_sc));
                            if constexpr (I8) {
                                l_run[u] += p;
                                s[u][kt][i] = p * w[kt][i];
                                top = fmaxf(top, fabsf(s[u][kt][i]));
                            } else {
                                pb[u][kt * 4 + i] = (M)p;
                            }
                        }
                    if constexpr (I8) {
                        if (any_moves || __any(top > unit[u].largest())) {
                            top = across<32>(across<16>(top, Max()), Max());
                            float f = 1.f;
                            if (moves || top > unit[u].largest()) f = unit[u].follow(alpha, top);
#pragma unroll
                            for (int e = 0; e < ET; ++e) o[u][e] *= f;
                        }
                        const float inv = unit[u].inverse();
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                pb[u][kt * 4 + i] = (M)(s[u][kt][i] * inv);
                                if constexpr (PAIRS) rest[u][kt * 4 + i] = (M)fmaf(s[u][kt][i], inv, -(float)pb[u][kt * 4 + i]);
                            }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) l_run[u] = add_pair<M>(__builtin_bit_cast(u32x4, pb[u])[i], l_run[u]);
                    }
                }
                if constexpr (!I8)
                    if (again && !all) {
                        constexpr uint32_t INF = std::is_same<M, _Float16>::value ? 0x7c00u : 0x7f80u;
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt) {
                            int seen = 0;   // of this lane's four slots, by any row
#pragma unroll
                            for (int u = 0; u < QT; ++u)
                                if (it_mask[kt] >> bit[u] & 1) seen = max(seen, len[u] - it_p0[kt] - 4 * g);
                            seen = row_max(seen);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
#pragma unroll
                                for (int w = 0; w < VW; ++w) {
                                    const uint32_t x = vreg[4 * kt + i][w], lo = (x & INF) == INF ? 0xffffu : 0u, up = (x >> 16 & INF) == INF ? 0xffff0000u : 0u;
                                    odd = odd || (i < seen && (lo | up));
                                    vreg[4 * kt + i][w] = x & ~(lo | up);
                                }
                        }
                    }
#pragma unroll
                for (int e = 0; e < ET; ++e) {
                    u32x4 w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (I8) w[i] = code_pair(vreg[2 * i][e >> 2], vreg[2 * i + 1][e >> 2], 0x0c040c00u + (e & 3) * 0x00010001u);
                        else w[i] = __builtin_amdgcn_perm(vreg[2 * i + 1][e >> 1], vreg[2 * i][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
                    }
                    const m8 vf = __builtin_bit_cast(m8, w);
#pragma unroll
                    for (int u = 0; u < QT; ++u) {
                        o[u][e] = Half<M>::mma(vf, pb[u], o[u][e]);
                        if constexpr (PAIRS) o[u][e] = Half<M>::mma(vf, rest[u], o[u][e]);
                    }
                }
                if (more) {
                    if (again) load_keys(at);
                    load_values(at);
                }
            }
            bool finite = true;
            if constexpr (!I8)
#pragma unroll
                for (int u = 0; u < QT; ++u)
#pragma unroll
                    for (int e = 0; e < ET; ++e)
#pragma unroll
                        for (int i = 0; i < 4; ++i) finite = finite && fabsf(o[u][e][i]) <= 3.4e38f;
            if (__builtin_expect(__all(finite), 1)) break;
        }

        // the waves' sums together: each brings its own to the common maximum
        odd = __any(odd);
        if (lane == 0) s_odd[wave] = odd;
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            l_run[u] = across<32>(across<16>(l_run[u], Add()), Add());
            if (g == 0) {
                s_m[wave][u * 16 + ql] = m_run[u];
                s_l[wave][u * 16 + ql] = l_run[u];
            }
        }
        __syncthreads();
        float m_all[QT], l_all[QT];
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            m_all[u] = kLowest;
#pragma unroll
            for (int w = 0; w < NW; ++w) m_all[u] = fmaxf(m_all[u], s_m[w][u * 16 + ql]);
            l_all[u] = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) l_all[u] += s_l[w][u * 16 + ql] * __builtin_amdgcn_exp2f((s_m[w][u * 16 + ql] - m_all[u]) * sc[u]);
            const float f = __builtin_amdgcn_exp2f((m_run[u] - m_all[u]) * sc[u]) * (I8 ? unit[u].R : 1.f);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < ET; e += 4) {
                    const float4 x = make_float4(o[u][e][i] * f, o[u][e + 1][i] * f, o[u][e + 2][i] * f, o[u][e + 3][i] * f);
                    *(float4*)&s_o[wave][u][i][lane][e] = x;
                }
        }
        __syncthreads();
        // wave i takes elements ET * (4g + i) .. of every row: ET neighbours per lane
        const int e0 = ET * (4 * g + wave);
        float x[QT][ET];
#pragma unroll
        for (int u = 0; u < QT; ++u)
#pragma unroll
            for (int e = 0; e < ET; ++e) {
                x[u][e] = 0.f;
#pragma unroll
                for (int w = 0; w < NW; ++w) x[u][e] += s_o[w][u][wave][lane][e];
            }
        if constexpr (!I8)
            if (__builtin_expect(s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3], 0))   // the values that counted as 0, to the rows that see them
                for (int i = i0; i < i1; i += 2) {
                    PageItem two[2] = {group_item(a, j, row0, len0, i), PageItem{0, 0, 0u, 0}};
                    if (i + 1 < i1) two[1] = group_item(a, j, row0, len0, i + 1);
                    if (two[0].full & two[1].full) continue;
                    for (const PageItem& one : two)
#pragma unroll
                        for (int u = 0; u < QT; ++u) {
                            const int seen = one.mask >> bit[u] & 1 ? min(len[u] - one.p0, 16) : 0;
                            for (int slot = 0; slot < seen; ++slot) {
                                const C* v = (const C*)V + (slot_of(one.page, one.p0) + slot) * HD + e0;
#pragma unroll
                                for (int e = 0; e < ET; ++e)
                                    if (!(fabsf((float)v[e]) <= 3.4e38f)) x[u][e] += (float)v[e];
                            }
                        }
                }
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            const int r = u * 16 + ql;
            if (r >= n_rows) continue;
            if (!whole) {
                float* to = part + (size_t)r * (HD + 4);
#pragma unroll
                for (int e = 0; e < ET; e += 4) *(float4*)(to + e0 + e) = make_float4(x[u][e], x[u][e + 1], x[u][e + 2], x[u][e + 3]);
                if (wave == 0 && g == 0) *(float2*)(to + HD) = make_float2(part_top(m_all[u] * sc[u]), l_all[u]);
            } else {
                const float inv = l_all[u] != 0.f ? 1.f / l_all[u] : 0.f;   // a row that sees nothing gets zeros
#pragma unroll
                for (int e = 0; e < ET; ++e) x[u][e] *= inv;
                page_store<T, ET>(a, j * a.group + bit[u], h * G + r0 + r - bit[u] * G, e0, x[u]);
            }
        }
    };

    if constexpr (!DEALT) {
        const int j = blockIdx.z, hb = blockIdx.x, k = blockIdx.y, count = group_items(a, j), n = page_parts(count, a.parts);
        if (k >= n) return;
        piece(j, hb, page_cut(count, k, n), page_cut(count, k + 1, n), n == 1, a.part + (((size_t)j * units + hb) * a.parts + k) * ROWS * (HD + 4));
    } else {
        const int w = blockIdx.x;
        if (w < n_groups && group_items(a, w) == 0)   // groups that see nothing are nobody's part
            for (int e = t; e < a.group * a.heads * (HD / 8); e += 256) {
                const int r = e / (HD / 8);
                const float zero[8] = {};
                page_store<T, 8>(a, w * a.group + r / a.heads, r % a.heads, e % (HD / 8) * 8, zero);
            }
        const PageShare sh = page_share(a, units, n_groups);
        PageNotes* notes = (PageNotes*)a.notes;
        if (w == 0 && t == 0) notes->cuts = sh.cuts;
        if (sh.j < 0) return;
        const int large = uniform(sh.cuts.large_of(sh.count)), n = large + uniform(sh.cuts.small_of(sh.count)), unit = sh.j * units + sh.hb;
        if (sh.k == 0 && large > 0 && t == 0) notes->first[unit].x = w;
        if (sh.k == large && t == 0) notes->first[unit].y = w;
        int i0, i1;
        sh.cuts.part(sh.count, sh.k, &i0, &i1);
        piece(sh.j, sh.hb, uniform(i0), uniform(i1), n == 1, a.part + (size_t)w * ROWS * (HD + 4));
    }
}

// Adds up the parts of the blockIdx.x-th unit, which lie behind each other.  A workgroup takes as
// many rows as it has groups of HD / 4 lanes; with fewer rows the groups share out a row's parts.  Loads of four parts at a time: the time is that of
// their latencies.
template <int HD, typename T, int QT>
__global__ __launch_bounds__(256) void k_page_join(PageAttentionArgs a)
{
    constexpr int LPG = HD / 4, GROUPS = 256 / LPG, ROWS = 16 * QT;
    __shared__ float s_m[GROUPS], s_l[GROUPS];
    __shared__ float4 s_x[GROUPS][LPG];
    const int unit = blockIdx.x, n_kv = a.p.n_kv, G = a.heads / n_kv, units = n_kv * a.row_blocks, j = unit / units, hb = unit % units;
    const int count = group_items(a, j);
    const PageNotes* notes = (const PageNotes*)a.notes;
    int n = page_parts(count, a.parts), large = 0, first_large = 0, first_small = unit * a.parts;
    if (a.parts == 0) {
        const PageCuts cuts = notes->cuts;
        large = cuts.large_of(count);
        n = large + cuts.small_of(count);
        first_large = notes->first[unit].x;
        first_small = notes->first[unit].y;
    }
    if (n < 2) return;
    const int group = threadIdx.x / LPG, e = threadIdx.x % LPG, first = blockIdx.y * GROUPS;
    const int rb = hb / n_kv, h = hb - rb * n_kv, r0 = rb * ROWS;
    const int n_rows = min(min(a.group * G - r0, ROWS) - first, GROUPS);
    if (n_rows <= 0) return;
    int sharers = 1;
    while (2 * sharers * n_rows <= GROUPS) sharers *= 2;
    const int r = first + group / sharers, turn = group % sharers;
    const bool there = group / sharers < n_rows;
    float m = kLowest, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float m_k, float l_k, const float4& y) {
        const float m_new = fmaxf(m, m_k), f = __builtin_amdgcn_exp2f(m - m_new), f_k = __builtin_amdgcn_exp2f(m_k - m_new);
        m = m_new;
        l = l * f + l_k * f_k;
        x[0] = x[0] * f + y.x * f_k;
        x[1] = x[1] * f + y.y * f_k;
        x[2] = x[2] * f + y.z * f_k;
        x[3] = x[3] * f + y.w * f_k;
    };
    if (there)
        for (int k = turn; k < n; k += 4 * sharers) {
            float4 y[4];
            float2 ml[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int part = min(k + i * sharers, n - 1);
                const float* q = a.part + ((size_t)(part < large ? first_large + part : first_small + part - large) * ROWS + r) * (HD + 4);
                y[i] = *(const float4*)(q + 4 * e);
                ml[i] = *(const float2*)(q + HD);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (k + i * sharers < n) add(ml[i].x, ml[i].y, y[i]);
        }
    s_x[group][e] = make_float4(x[0], x[1], x[2], x[3]);
    if (e == 0) {
        s_m[group] = m;
        s_l[group] = l;
    }
    __syncthreads();
    if (!there || turn > 0) return;
    for (int k = 1; k < sharers; ++k) add(s_m[group + k], s_l[group + k], s_x[group + k][e]);
    const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= inv;
    const int b = (r0 + r) / G;
    page_store<T, 4>(a, j * a.group + b, h * G + r0 + r - b * G, 4 * e, x);
}

// ------------------------------------------------------------------------------------------ fork
// Three launches, or one (k_pages_fork_few).  Claims: of each page the lowest row of `to` that writes into it, -1 if a row holds it that does not (or somebody else
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

constexpr int kForkThreads = 1024, kForkPages = 4096;   // pages of a workgroup

// Counts, over all n entries of a list (16-byte aligned), those that f takes: this thread's four of the kForkPages from `first` on, its
// share of those before `first`, and of all.  Four loads at a time.
struct Counts {
    int mine, ahead, every;
};
template <typename F>
__device__ __forceinline__ Counts count_pages(const int32_t* list, int n, int first, F f)
{
    Counts c{0, 0, 0};
    constexpr int AT_ONCE = 4;
    for (int p0 = 0; p0 < n; p0 += AT_ONCE * kForkPages) {
        int x[AT_ONCE][4];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int p = p0 + u * kForkPages + 4 * (int)threadIdx.x;
            if (p + 3 < n) {
                const int4 v = *(const int4*)(list + p);
                x[u][0] = v.x, x[u][1] = v.y, x[u][2] = v.z, x[u][3] = v.w;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) x[u][k] = p + k < n ? list[p + k] : 0;
            }
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int at = p0 + u * kForkPages, p = at + 4 * (int)threadIdx.x;
            int here = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) here += p + k < n && f(x[u][k], p + k);
            c.every += here;
            if (at < first) c.ahead += here;
            if (at == first) c.mine = here;
        }
    }
    return c;
}

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
    const Counts c = count_pages(a.claim, n, first, [](int x, int) { return x == kFree; });
    const int every = Scan<kForkThreads>(c.every, s_scan).all, ahead = Scan<kForkThreads>(c.ahead, s_scan).all;
    int rank = ahead + Scan<kForkThreads>(c.mine, s_scan).before;
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

// The same in one workgroup, with the claims in LDS: where rows and pages are few the three launches are most of the time.  Bound by the chain parent,
// length, entries, needs, pages: 6.8 us for 32 rows of 110 entries (three launches 13), 9.8 for 512 of 18.
constexpr int kFewRowsOfTable = 1024, kFewPages = 16384;   // of one workgroup
template <typename A>
__device__ __forceinline__ int entry_row(int e, const A& t) { return (int)((uint32_t)e / (uint32_t)t.stride); }

__global__ __launch_bounds__(kForkThreads) void k_pages_fork_few(ForkArgs a)
{
    extern __shared__ __attribute__((aligned(16))) int s_claim[];   // [n_pages, in whole fours of a thread]
    __shared__ int s_start[kFewRowsOfTable], s_parent[kFewRowsOfTable], s_held[kFewRowsOfTable], s_last[kFewRowsOfTable], s_source[kFewRowsOfTable];
    __shared__ int s_scan[kForkThreads / 64 + 1];
    const int rows = a.to.rows, n = a.to.n_pages, t = threadIdx.x, per = (n + 4 * kForkThreads - 1) / (4 * kForkThreads) * 4;
    int wanted = 0;
    if (t < rows) {
        const Fork f(a, t);
        s_parent[t] = f.parent;
        s_held[t] = f.held;
        s_last[t] = f.last;
        s_source[t] = -1;
        wanted = f.wanted - f.held;
        a.to.lengths[t] = f.new_len;
        a.src[t] = a.dst[t] = -1;
    }
    for (int p = t; p < per * kForkThreads; p += kForkThreads) s_claim[p] = p >= n || (a.held && a.held[p]) ? -1 : kFree;
    __syncthreads();
    constexpr int AT_ONCE = 4;
    const int entries = rows * a.to.stride;
    for (int e0 = t; e0 < entries; e0 += AT_ONCE * kForkThreads) {
        int row[AT_ONCE], entry[AT_ONCE], page[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int e = min(e0 + u * kForkThreads, entries - 1);
            row[u] = entry_row(e, a.to);
            entry[u] = e - row[u] * a.to.stride;
            page[u] = -1;
            if (entry[u] < s_held[row[u]]) page[u] = a.from.pages[(int64_t)s_parent[row[u]] * a.from.stride + entry[u]];
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            if (e0 + u * kForkThreads >= entries) break;
            const bool there = is_page(a.from, page[u]), last = entry[u] == s_last[row[u]];
            if (there) atomicMin(&s_claim[page[u]], last ? row[u] : -1);
            if (there && last) s_source[row[u]] = page[u];
            a.to.pages[e0 + u * kForkThreads] = there ? page[u] : -1;
        }
    }
    __syncthreads();   // which also has the entries written before some of them are written again
    const bool copies = t < rows && s_source[t] >= 0 && s_claim[s_source[t]] != t;
    const Scan<kForkThreads> need(t < rows ? wanted + copies : 0, s_scan);
    if (t < rows) {
        s_start[t] = need.before;
        if (!copies) s_source[t] = -1;
    }
    const int4* mine = (const int4*)(s_claim + t * per);
    int free_here = 0;
    for (int k = 0; k < per / 4; ++k) free_here += (mine[k].x == kFree) + (mine[k].y == kFree) + (mine[k].z == kFree) + (mine[k].w == kFree);
    const Scan<kForkThreads> free_pages(free_here, s_scan);
    __syncthreads();
    auto give = [&](int rank, int page) {   // as in k_pages_hand_out
        int lo = 0, hi = rows - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (s_start[mid] <= rank) lo = mid;
            else hi = mid - 1;
        }
        const int shared = s_source[lo], k = rank - s_start[lo] - (shared >= 0);
        a.to.pages[(int64_t)lo * a.to.stride + (k < 0 ? s_last[lo] : s_held[lo] + k)] = page;
        if (k < 0 && page >= 0) {
            a.src[lo] = shared;
            a.dst[lo] = page;
        }
    };
    if (free_here > 0 && free_pages.before < need.all) {
        int rank = free_pages.before;
        for (int k = 0; k < per && rank < need.all; ++k)
            if (s_claim[t * per + k] == kFree) give(rank++, t * per + k);
    }
    for (int k = free_pages.all + t; k < need.all; k += kForkThreads) give(k, -1);
    if (t == 0) *a.missing = max(need.all - free_pages.all, 0);
}

// ------------------------------------------------------------------------------------------ compact
// Four launches, or one (k_pages_compact_few): which pages are in use; how many before each, so that the k-th that has to move and the k-th hole below
// meet at k; tables and places by that.  The counting reads the whole list in every workgroup (26521 pages 11 us, half a million would take
// 100: then blocks of it would have to be counted first).
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
    const Counts c = count_pages(a.used, n, first, [](int x, int) { return x != 0; });
    const int every = Scan<kForkThreads>(c.every, s_scan).all, ahead = Scan<kForkThreads>(c.ahead, s_scan).all;
    // pages in use that keep their numbers
    const int below = Scan<kForkThreads>(count_pages(a.used, every, 0, [](int x, int) { return x != 0; }).every, s_scan).all;
    const int moves = every - below;
    int used_before = ahead + Scan<kForkThreads>(c.mine, s_scan).before;
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

// The same in one workgroup, as k_pages_fork_few.
__global__ __launch_bounds__(kForkThreads) void k_pages_compact_few(CompactArgs a)
{
    extern __shared__ __attribute__((aligned(16))) int s_place[];   // [n_pages, in whole fours of a thread]: in use or not, then the new number
    __shared__ int s_hole[kFewPages / 4], s_len[kFewRowsOfTable], s_scan[kForkThreads / 64 + 1];
    const int rows = a.from.rows, n = a.from.n_pages, t = threadIdx.x, per = (n + 4 * kForkThreads - 1) / (4 * kForkThreads) * 4;
    if (t < rows) {
        s_len[t] = row_length(a.from, t);
        a.to.lengths[t] = s_len[t];
    }
    for (int p = t; p < per * kForkThreads; p += kForkThreads) s_place[p] = p < n && a.held && a.held[p];
    __syncthreads();
    constexpr int AT_ONCE = 4;
    const int entries = rows * a.from.stride;
    auto page_at = [&](int e) {
        const int row = entry_row(e, a.from);
        if ((e - row * a.from.stride) * a.from.page >= s_len[row]) return -1;
        const int p = a.from.pages[e];
        return is_page(a.from, p) ? p : -1;
    };
    auto every = [&](auto f) {   // f(entry, page), some loads at a time
        for (int e0 = t; e0 < entries; e0 += AT_ONCE * kForkThreads) {
            int page[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) page[u] = page_at(min(e0 + u * kForkThreads, entries - 1));
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (e0 + u * kForkThreads < entries) f(e0 + u * kForkThreads, page[u]);
        }
    };
    every([&](int, int p) {
        if (p >= 0) s_place[p] = 1;
    });
    __syncthreads();
    const int first = t * per;
    int used_here = 0;
    for (int k = 0; k < per; k += 4) {
        const int4 x = *(const int4*)(s_place + first + k);
        used_here += (x.x + x.y) + (x.z + x.w);
    }
    const Scan<kForkThreads> used(used_here, s_scan);
    int below_here = 0;   // pages in use that keep their numbers
    for (int k = 0; k < per && first + k < used.all; ++k) below_here += s_place[first + k];
    const Scan<kForkThreads> below(below_here, s_scan);
    const int moves = used.all - below.all;
    int before = used.before;
    for (int k = 0; k < per && first + k < used.all; ++k) {
        const int p = first + k;
        if (s_place[p]) ++before;
        else {
            s_hole[p - before] = p;
            a.dst[p - before] = p;
        }
    }
    __syncthreads();
    before = used.before;
    for (int k = 0; k < per && first + k < n; ++k) {
        const int p = first + k;
        int to = -1;
        if (s_place[p]) {
            to = p;
            if (p >= used.all) {
                const int rank = before - below.all;
                to = s_hole[rank];
                a.src[rank] = p;
            }
            ++before;
        }
        s_place[p] = to;
        if (p >= moves && p < n / 2) a.src[p] = a.dst[p] = -1;
    }
    if (t == 0) {
        a.counts[0] = used.all;
        a.counts[1] = moves;
    }
    __syncthreads();
    every([&](int e, int p) { a.to.pages[e] = p >= 0 ? s_place[p] : -1; });
    if (a.place)
        for (int p = t; p < n; p += kForkThreads) a.place[p] = s_place[p];
}

// ------------------------------------------------------------------------------------------ copies
constexpr int kCopyLayers = 32, kCopyPairs = 2048;   // of a launch
struct CopyArgs {
    void* p[kCopyLayers][2];
    float* scale[kCopyLayers][2];
    const int32_t *src, *dst, *count;
    int n, n_pages;
    int64_t bytes, scale_bytes;   // of a page
};

// A workgroup takes a piece of kCopyPiece bytes of a page's keys or values (the first one the scales too) in one layer, of every gridDim.x-th pair.  All
// loads of a piece are issued before its first store.  Bound by the bytes: rows that get copies of the same page are neighbours, so its second reader
// finds it in a cache, and what is written goes past them (512 rows and 24 layers 67 us, 1.7 GB of a compaction 325; reads past the caches too 77, 320; written
// into them 70, 349).
constexpr int kCopyAtOnce = 4, kCopyPiece = kCopyAtOnce * 256 * 16;
__global__ __launch_bounds__(256) void k_pages_copy(CopyArgs a)
{
    const int layer = blockIdx.y >> 1, which = blockIdx.y & 1;
    const int n = a.count ? min(a.n, *a.count) : a.n;
    const int64_t k0 = (int64_t)blockIdx.z * kCopyPiece + threadIdx.x * 16;
    for (int i = blockIdx.x; i < n; i += gridDim.x) {
        const int s = a.src[i], d = a.dst[i];
        if (s < 0 || s >= a.n_pages || d < 0 || d >= a.n_pages || s == d) continue;
        const char* from = (const char*)a.p[layer][which] + s * a.bytes;
        char* to = (char*)a.p[layer][which] + d * a.bytes;
        u32x4 x[kCopyAtOnce];
#pragma unroll
        for (int u = 0; u < kCopyAtOnce; ++u)
            if (k0 + u * 4096 < a.bytes) x[u] = *(const u32x4*)(from + k0 + u * 4096);
#pragma unroll
        for (int u = 0; u < kCopyAtOnce; ++u)
            if (k0 + u * 4096 < a.bytes) __builtin_nontemporal_store(x[u], (u32x4*)(to + k0 + u * 4096));
        if (!a.scale_bytes || blockIdx.z > 0) continue;
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
    if (a.group > 1) k_page_items<<<a.n / a.group, kItemThreads, 0, s>>>(a);
    auto go = [&](auto dim, auto t, auto e, auto tiles) {
        constexpr int HD = decltype(dim)::value, QT = decltype(tiles)::value;
        typedef decltype(t) T;
        typedef decltype(e) C;
        const int units = a.p.n_kv * a.row_blocks, groups = a.n / a.group;
        if (a.parts > 0) k_attention_pages<HD, T, C, QT, false><<<dim3(units, a.parts, groups), 256, 0, s>>>(a);
        else k_attention_pages<HD, T, C, QT, true><<<page_grid(a.at_once, units * groups, a.group), 256, 0, s>>>(a);
        if (a.parts != 1) k_page_join<HD, T, QT><<<dim3(units * groups, 16 * QT * HD / 1024), 256, 0, s>>>(a);
    };
    with_types(a.p.hd, token, a.p.dtype, [&](auto dim, auto t, auto e) {
        typedef decltype(t) T;
        typedef decltype(e) C;
        if constexpr (std::is_same<C, int8_t>::value || std::is_same<C, T>::value) {
            if (a.tiles == 1) go(dim, t, e, std::integral_constant<int, 1>{});
            else go(dim, t, e, std::integral_constant<int, 2>{});
        }
    });
}

// Whether one workgroup does it: what its 1024 threads take one after another costs more than two or three launches from some number of entries on.  Three
// launches / one (us, with a copy of 5 behind them, graphs): forks of 32 rows of 110 entries 16.7 / 10.0, 20 of 950 15.3 / 11.4, 512 of 50 19.7 / 17.0, 256 of 133
// 17.8 / 22.8, 1024 of 50 22.4 / 27.9.  Compactions, which go through the entries twice, 24 rows of 60 15.2 / 9.7, 64 of 150 18.3 / 16.2, 200 of 65 19.3 /
// 19.5, 20 of 950 and 12000 pages 25.4 / 33.7.
static bool pages_few(int n_pages, int rows, int stride, int most_pages, int most_entries)
{
    return rows <= kFewRowsOfTable && n_pages <= most_pages && (int64_t)rows * stride <= most_entries;
}

void launch_pages_fork(const ForkArgs& a, hipStream_t s)
{
    const int n = a.to.n_pages;
    if (pages_few(n, a.to.rows, a.to.stride, kFewPages, 28000)) {
        k_pages_fork_few<<<1, kForkThreads, (size_t)(n + 4 * kForkThreads - 1) / (4 * kForkThreads) * (16 * kForkThreads), s>>>(a);
        return;
    }
    k_pages_claims<<<(n + 255) / 256, 256, 0, s>>>(a.claim, a.held, n);
    if (a.to.rows > 0) k_pages_inherit<<<a.to.rows, 256, 0, s>>>(a);
    k_pages_hand_out<<<(n + kForkPages - 1) / kForkPages, kForkThreads, (size_t)(a.to.rows + 1) * 4, s>>>(a);
}

void launch_pages_compact(const CompactArgs& a, hipStream_t s)
{
    const int n = a.from.n_pages;
    if (pages_few(n, a.from.rows, a.from.stride, kFewPages / 2, 12000)) {
        k_pages_compact_few<<<1, kForkThreads, (size_t)(n + 4 * kForkThreads - 1) / (4 * kForkThreads) * (16 * kForkThreads), s>>>(a);
        return;
    }
    k_pages_unused<<<(n + 255) / 256, 256, 0, s>>>(a.used, a.held, n);
    if (a.from.rows > 0) k_pages_mark<<<a.from.rows, 256, 0, s>>>(a);
    k_pages_rank<<<(n + kForkPages - 1) / kForkPages, kForkThreads, 0, s>>>(a);
    if (const int blocks = a.from.rows + (a.place ? (n + 255) / 256 : 0)) k_pages_renumber<<<blocks, 256, 0, s>>>(a);
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
        k_pages_copy<<<dim3(n < kCopyPairs ? n : kCopyPairs, 2 * here, (unsigned)((a.bytes + kCopyPiece - 1) / kCopyPiece)), 256, 0, s>>>(a);
    }
}

}  // namespace ss

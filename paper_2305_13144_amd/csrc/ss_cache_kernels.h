// Kernels of the operators on device tensors: a key/value cache in 8 or 16 bits, the attention of single tokens or of drafted
// trees over it, and the causal attention of packed prompts.  Included by ss_kernels.hip.
#ifndef SS_CACHE_KERNELS_H
#define SS_CACHE_KERNELS_H

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "ss_device.h"
#include "ss_plan.h"

namespace ss {

// ------------------------------------------------------------------------------------------ element types
// T: _Float16 or __bf16.  Operands of the matrix instructions are 8 of them per lane.
template <typename T>
struct Half;
template <>
struct Half<_Float16> {
    typedef f16x8 x8;
    static __device__ __forceinline__ f32x4 mma(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
template <>
struct Half<__bf16> {
    typedef bf16x8 x8;
    static __device__ __forceinline__ f32x4 mma(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

constexpr float kLowest = -3.0e38f;   // running maximum of no score: finite, so that exp2(-inf - kLowest) is 0

// Eight values of 16 bits as floats, and back (half saturates at its largest finite value, NaN stays NaN).
template <typename T>
__device__ __forceinline__ void to_floats(const u32x4& r, float (&f)[8])
{
    const typename Half<T>::x8 h = __builtin_bit_cast(typename Half<T>::x8, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)h[i];
}
template <typename T>
__device__ __forceinline__ u32x4 from_floats(const float (&f)[8])
{
    typename Half<T>::x8 h;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (std::is_same<T, _Float16>::value) h[i] = __builtin_bit_cast(_Float16, f2h(f[i]));
        else h[i] = (__bf16)f[i];
    }
    return __builtin_bit_cast(u32x4, h);
}

// What a weight's exponent s * sc takes off, of the maximum m that the weights are relative to.  Its rounding, up to 2^-24 of it, is a
// factor common to all of a row's slots, but where it is large no factor that a weight can hold (from 2^28 on half's range is left, from 2^31
// on the exponential's): there the differences are formed first.  A branch of the wave that ordinary scores never take.
template <typename V, int N>
__device__ __forceinline__ float exponent_top(float m, float sc, V (&s)[N])
{
    float top = fmaxf(m * sc, kLowest);
    if (__any(fabsf(top) > 0x1p22f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] -= m;
        top = 0.f;
    }
    return top;
}

// score - top, where the score is a product.  Both are to be the rounded numbers: with the product inside the difference (one fma) its rounding,
// which is in the top, would remain of the largest score.
__device__ __forceinline__ float below_top(float score, float top)
{
#pragma clang fp contract(off)
    return score - top;
}

// The power of two that brings a row whose largest magnitude is `top` (in bf16) to 2^14 to 2^15, and its inverse.  2^-100 and less count as that.
__device__ __forceinline__ float half_power(float top, float* inverse)
{
    const int ex = max((int)(__float_as_uint(top) >> 23) - 127, -100);   // top is below 2^(ex + 1)
    *inverse = __uint_as_float((uint32_t)(127 - 14 + ex) << 23);
    return __uint_as_float((uint32_t)(127 + 14 - ex) << 23);
}

// R of a row over an 8-bit cache.  The largest product top = p * scale that the row has met is at least 2^6 R, and a product up to 2^15 R
// is held without a change of R: half's largest number is 2^16, and what rounds in its subnormals is off by at most 2^-25 R, 2^-31 of the
// largest.  Where the weights' maximum has moved (by `alpha`), R moves with it, as the products that it was made for no longer count.
struct WeightUnit {
    float R = 0.f;
    __device__ __forceinline__ float largest() const { return R * 0x1p15f; }
    __device__ __forceinline__ float inverse() const { return __uint_as_float(0x7f000000u - __float_as_uint(R)); }
    // `top`: of the products that come; returns what the sums so far, in the old unit, are to be multiplied by
    __device__ __forceinline__ float follow(float alpha, float top)
    {
        const float old = R * alpha;
        const uint32_t two = __float_as_uint(fmaxf(old * 64.f, top)) & 0x7f800000u;
        const uint32_t bits = min(max(two, 7u << 23) - (6u << 23), 0x7e800000u);   // 2^-126 to 2^126
        R = __uint_as_float(bits);
        return old * inverse();
    }
};

// A chunk's maximum as it is kept for the join: finite, so that differences are numbers.
__device__ __forceinline__ float part_top(float m) { return fminf(fmaxf(m, kLowest), -kLowest); }

// First slot's vector of head h of sequence i in a cache, or -1 if the tables do not describe a slab inside it.
__device__ __forceinline__ int64_t slab_of(const CacheView& c, int i, int* slots)
{
    const int64_t at = c.start[i];
    const int n = c.slots[i];
    *slots = n;
    return slab_inside(at, n, c.total) ? at * c.n_kv : -1;
}

// ------------------------------------------------------------------------------------------ cache: write and read
// A vector of HD elements is HD / 8 neighbouring lanes', 16 bytes each.  A workgroup takes 16 tokens through kCachePasses passes over 128 / HD
// heads, keys and values in different workgroups: tokens of a prompt are neighbours in the cache, so that a head's vectors leave
// as runs of 16 (with a token's heads side by side instead 8745 tokens of 32 heads of 128 took 64 us to write and 54 to read).
constexpr int kCachePasses = 4, kCacheTokens = 16;

// Of a lane: its token, that token's first vector in the cache (-1: none) and slots between heads, its first head.
struct CachePlace {
    int t, slots, head;
    int64_t at;
    static constexpr int step(int hd) { return 128 / hd; }   // heads of a pass
    __device__ __forceinline__ CachePlace(const CacheView& c, const int32_t* seq, const int32_t* slot, int n, int vector, int hd)
    {
        t = blockIdx.x * kCacheTokens + vector % kCacheTokens;
        head = blockIdx.y * (kCachePasses * step(hd)) + vector / kCacheTokens;
        at = -1;
        slots = 0;
        if (t >= n) return;
        const int s = seq[t], place = slot[t];
        if (s < 0 || s >= c.n_seq) return;
        const int64_t base = slab_of(c, s, &slots);
        if (base >= 0 && place >= 0 && place < slots) at = base + place;
    }
};

// Largest magnitude in a vector as the bits of a float: those are ordered as the numbers, with infinities and NaN on top.
template <int HD>
__device__ __forceinline__ uint32_t vector_top(uint32_t m)
{
    auto top = [&](float o) { const uint32_t u = __float_as_uint(o); m = m > u ? m : u; };
    top(dpp<kDppXor1>(__uint_as_float(m)));
    top(dpp<kDppXor2>(__uint_as_float(m)));
    top(dpp<kDppHalfMirror>(__uint_as_float(m)));
    if (HD == 128) top(dpp<kDppMirror>(__uint_as_float(m)));
    return m;
}

// A vector in 8 bits: scale = max|x| / 127 and code = x / scale, both divisions and the step to a whole number rounded to
// nearest (even), as written.  x times the reciprocal is within 127 * 2^-23 < 1.6e-5 of that quotient, and the quotient's own rounding
// moves it by at most 2^-18, so only where a product is that near to the middle of two codes are quotients formed.  The whole
// number is the low byte of the product plus 3 * 2^22.  A vector with an infinity or NaN gets the scale NaN (it is read back as NaN
// throughout, by those who read it), one of zeros the scale 0.
template <int HD>
__device__ __forceinline__ float quantise(const float (&x)[8], uint2* codes)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = __float_as_uint(x[i]) & 0x7fffffffu;
        m = m > u ? m : u;
    }
    m = vector_top<HD>(m);
    const float scale = m < 0x7f800000u ? __uint_as_float(m) / 127.f : __uint_as_float(0x7fc00000u);
    const bool plain = scale > 0x1p-100f;   // not 0, not NaN, and its reciprocal a normal number
    const float inv = 1.f / scale;
    constexpr float kWhole = 12582912.f;
    uint32_t code[8];
    float off = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = x[i] * inv, r = y + kWhole;
        off = fmaxf(off, fabsf(y - (r - kWhole)));
        code[i] = __float_as_uint(r);
    }
    if (__any(!plain || off > 0.49998f)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float r = scale > 0.f ? fminf(fmaxf(rintf(x[i] / scale), -127.f), 127.f) : 0.f;
            code[i] = (uint32_t)(int)r;
        }
    }
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(code[4 * i + 1], code[4 * i], 0x0c0c0400u), up = __builtin_amdgcn_perm(code[4 * i + 3], code[4 * i + 2], 0x04000c0cu);
        w[i] = lo | up;
    }
    *codes = make_uint2(w[0], w[1]);
    return scale;
}

__device__ __forceinline__ void codes_to_floats(const uint2& c, float scale, float (&f)[8])
{
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)((int)(w[i >> 2] << (24 - 8 * (i & 3))) >> 24) * scale;
}

// TOKEN: type of the tokens' rows; CACHE: int8_t, _Float16 or __bf16.
// Bound by the bytes: 2 in and 1 out per element.  All loads of a workgroup's passes are issued before the first is used, past the
// caches: they are used once (8745 tokens of 32 heads of 128, written and read: 96 -> 91 us).
template <int HD, typename TOKEN, typename CACHE>
__global__ __launch_bounds__(256) void k_cache_write(CacheView c, RowsView k, RowsView v, const int32_t* __restrict__ seq,
                                                     const int32_t* __restrict__ slot, int n)
{
    constexpr int LPV = HD / 8, STEP = CachePlace::step(HD);
    const bool values = blockIdx.z;
    const RowsView src = values ? v : k;
    const int part = threadIdx.x % LPV;
    const CachePlace at(c, seq, slot, n, threadIdx.x / LPV, HD);
    u32x4 in[kCachePasses];
    int64_t to[kCachePasses];
#pragma unroll
    for (int p = 0; p < kCachePasses; ++p) {   // beyond the last token or head: read again, written nowhere
        const int h = at.head + p * STEP;
        in[p] = __builtin_nontemporal_load((const u32x4*)((const TOKEN*)src.p + (int64_t)min(at.t, n - 1) * src.row + (int64_t)min(h, c.n_kv - 1) * src.head + part * 8));
        to[p] = at.at >= 0 && h < c.n_kv ? at.at + (int64_t)h * at.slots : -1;
    }
#pragma unroll
    for (int p = 0; p < kCachePasses; ++p) {
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
__global__ __launch_bounds__(256) void k_cache_read(CacheView c, RowsView k, RowsView v, const int32_t* __restrict__ seq,
                                                    const int32_t* __restrict__ slot, int n)
{
    constexpr int LPV = HD / 8, STEP = CachePlace::step(HD);
    const bool values = blockIdx.z;
    const RowsView dst = values ? v : k;
    const int part = threadIdx.x % LPV;
    const CachePlace at(c, seq, slot, n, threadIdx.x / LPV, HD);
    if (at.at < 0) return;
    u32x4 in[kCachePasses];
    float scale[kCachePasses];
    TOKEN* to[kCachePasses];
#pragma unroll
    for (int p = 0; p < kCachePasses; ++p) {
        const int h = at.head + p * STEP;
        to[p] = nullptr;
        if (h >= c.n_kv) continue;
        const int64_t from = at.at + (int64_t)h * at.slots;
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
    for (int p = 0; p < kCachePasses; ++p) {
        if (!to[p]) continue;
        if constexpr (std::is_same<CACHE, TOKEN>::value) {
            *(u32x4*)to[p] = in[p];
        } else {
            float x[8];
            if constexpr (std::is_same<CACHE, int8_t>::value) codes_to_floats(make_uint2(in[p][0], in[p][1]), scale[p], x);
            else to_floats<CACHE>(in[p], x);
            __builtin_nontemporal_store(from_floats<TOKEN>(x), (u32x4*)to[p]);   // 91 -> 76 us with the writes above: they stay in L2
        }
    }
}

// The engine's way into the cache.  As k_rope_append: row j's sums of q|k|v, whose columns are in the order of qkv_col, rotated at its
// position; here a vector is HD / 8 lanes', 4 elements of each half per lane.  Keys and values are coded from their fp32 values.
// Bound by its bytes (fp32 slices in, halves and codes out) and, in decode steps, by the launch: the codes need no pass of their own.
template <int HD, typename CACHE>
__global__ __launch_bounds__(256) void k_rotate_store(MbState st, const float* __restrict__ part, int ksplit, size_t part_stride,
                                                      const float* __restrict__ rcos, const float* __restrict__ rsin, f16_t* __restrict__ rows,
                                                      int dense_kv, CacheView c, const int32_t* __restrict__ slot, int d)
{
    constexpr int LPV = HD / 8, VPP = 256 / LPV, MAX_SPLIT = 8;
    const int j = blockIdx.x, vec = blockIdx.y * VPP + threadIdx.x / LPV, e = threadIdx.x % LPV * 4;
    const int count = *st.d_n, seq = st.tr_row[j], pos = st.tr_pos[j], at = slot[j];
    if (j >= count || vec >= 3 * c.n_kv) return;
    const int which = vec / c.n_kv, h = vec - which * c.n_kv;   // 0 q, 1 k, 2 v
    const float* p = part + (size_t)j * 3 * d + which * d + h * HD + qkv_col(e);
    float4 a[MAX_SPLIT], b[MAX_SPLIT];   // every slice's loads before the first sum
#pragma unroll
    for (int s = 0; s < MAX_SPLIT; ++s)
        if (s < ksplit) {
            a[s] = *(const float4*)(p + s * part_stride);
            b[s] = *(const float4*)(p + s * part_stride + 16);
        }
    const float4 cs = *(const float4*)(rcos + (size_t)pos * (HD / 2) + e), sn = *(const float4*)(rsin + (size_t)pos * (HD / 2) + e);
#pragma unroll
    for (int s = 1; s < MAX_SPLIT; ++s)
        if (s < ksplit) {
            a[0] = make_float4(a[0].x + a[s].x, a[0].y + a[s].y, a[0].z + a[s].z, a[0].w + a[s].w);
            b[0] = make_float4(b[0].x + b[s].x, b[0].y + b[s].y, b[0].z + b[s].z, b[0].w + b[s].w);
        }
    float x[8] = {a[0].x, a[0].y, a[0].z, a[0].w, b[0].x, b[0].y, b[0].z, b[0].w};
    if (which < 2) {
        const float cc[4] = {cs.x, cs.y, cs.z, cs.w}, ss[4] = {sn.x, sn.y, sn.z, sn.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 r = rotated(x[i], x[i + 4], cc[i], ss[i]);
            x[i] = r.x;
            x[i + 4] = r.y;
        }
    }
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f2kv(x[2 * i]) | (uint32_t)f2kv(x[2 * i + 1]) << 16;
    if (which == 0 || dense_kv) {
        f16_t* to = rows + (size_t)j * 3 * d + which * d + h * HD + e;
        *(uint2*)to = make_uint2(w[0], w[1]);
        *(uint2*)(to + HD / 2) = make_uint2(w[2], w[3]);
    }
    if (which == 0) return;
    const int64_t to = c.start[seq] * c.n_kv + (int64_t)h * c.slots[seq] + at;
    CACHE* const vector = (CACHE*)(which == 1 ? c.k : c.v) + to * HD + e;
    if constexpr (std::is_same<CACHE, int8_t>::value) {
        uint2 codes;
        const float scale = quantise<HD>(x, &codes);
        *(uint32_t*)vector = codes.x;
        *(uint32_t*)(vector + HD / 2) = codes.y;
        if (e == 0) (which == 1 ? c.k_scale : c.v_scale)[to] = scale;
    } else {
        *(uint2*)vector = make_uint2(w[0], w[1]);
        *(uint2*)(vector + HD / 2) = make_uint2(w[2], w[3]);
    }
}

// ------------------------------------------------------------------------------------------ attention over a cache
// Rows of a unit: the (node, query head) pairs of one sequence and one key/value head, row r = node * G + (head within its
// group), G = query heads per key/value head; a decode step is the tree of one node.  A wave takes 16 * QT rows through steps of
// 32 slots with an online softmax in powers of two:
//   scores      S^T[slot][row] = K Q^T        K the A operand (16 slots x 32 elements), Q^T the B operand
//   weights     lane (row = lane % 16, g = lane / 16) holds slots 4g..4g+3 of both 16-slot tiles: the very B operand of
//   values      O^T[element][row] += V^T P^T  with its slots taken in that order; V^T's A operand holds, for element
//               ET * (lane % 16) + t of tile t, the same 8 slots, so a lane loads ET neighbouring elements of 8 slots (whole
//               cache lines per 16 lanes) and exchanges them in registers.
// Nothing is staged in LDS: a decode step uses each byte of the cache once, a tree of up to 32 rows too, and the rows beyond
// come back to it through L2 (their workgroups are neighbours on one die).  The four waves of a workgroup take turns
// over a unit's steps and join their sums through LDS at the end; a unit's slots are cut into chunks for as many workgroups as
// fill the chip (tree_plan), whose sums k_tree_join adds up.
// 8-bit caches: codes become halves exactly (1152 + code as a half's bits, less 1152), the key's scale multiplies the score
// and the value's the weight.  Weights are rounded to half, so they are held as w = p * scale / R with R a power of two that follows
// the largest p * scale of the row (WeightUnit): a slot of large values and no weight takes no bits from the others.  Their sum stays that of the
// unrounded p, as what is rounded has the scale in it, so that the rounding of a large weight does not cancel: each is off by half a step of half, 2^-11.
// Beside results in bf16 that is nothing.  Results in half of up to 16 rows take the weight as the sum of two halves, a second product for
// what the first leaves (relative error of a long row 0.00029 -> 0.00021, the result's own rounding; 64 rows of 32 heads at 3000 slots 106 -> 108 us,
// with heads of 64 60 -> 63); with more rows the vector work and the products bound it (40 -> 43 us in blocks of 32 rows, 46 -> 53 in the
// kernel for more), and their results keep the one rounding.  Over 16-bit caches a weight is rounded to the values' type, which the matrix instructions want
// of both operands (bf16: 2^-8 each, 0.0020 where the result's rounding makes 0.0016), and the sum is that of the rounded weights.  A row of bf16 queries is brought into half's range by a power of two of its own:
// exact down to 2^-31 of its largest element, 8 bits being fewer than 11.
// Slots that a row must not see weigh 0 whatever they hold: scores by selection; infinite and NaN values of steps that not every row sees
// count as 0 in the products and are added at the end to the rows that see them.
// Bound by the cache's bytes at long contexts (64 rows to 8000 slots, 32 heads on 8, 8 bits: 89 to 92 us, 5.7 TB/s but for 2552 chunks of unlike length), at short
// ones by a chain of latencies: table, slots, the second of two steps one behind the other, barriers, join (16 rows to 250 slots, 32 heads, halves: 12 us).  Operands are
// requested again as their registers fall free: 3 waves a SIMD, where a second set of registers leaves 2 and a fourth wave spills (98 -> 203 us).
template <typename C, typename T>
struct MathType { typedef T type; };           // 16-bit cache: its own type
template <typename T>
struct MathType<int8_t, T> { typedef _Float16 type; };

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// The j-th sequence of a call: its rows (nodes), its history, its slots (history and nodes, as far as the slab goes) and the first
// vector of its slab.  No rows where the tables leave the rows that there are, no slots where they leave the cache.
struct TreeSeq {
    int node0, n_nodes, ctx, len, slots;
    int64_t base;
};
__device__ __forceinline__ TreeSeq tree_sequence(const TreeArgs& a, int j)
{
    const CacheView& c = a.c;
    TreeSeq s{j, 0, 0, 0, 0, 0};
    // what does not depend on other tables is read at once
    int seq = j, end = j + 1;
    const int live = a.d_n ? *a.d_n : a.n_seq, own = min(j, c.n_seq - 1);
    int64_t at = c.start[own];
    s.slots = c.slots[own];
    s.ctx = max(a.context[j], 0);
    if (a.nodes) {
        s.node0 = a.nodes[j];
        end = a.nodes[j + 1];
    }
    if (a.seq) {
        seq = a.seq[j];
        const int there = min(max(seq, 0), c.n_seq - 1);
        at = c.start[there];
        s.slots = c.slots[there];
    }
    if (j < live) s.n_nodes = (int)table_rows(s.node0, end, a.max_nodes, a.q.rows);
    if (seq >= 0 && seq < c.n_seq && slab_inside(at, s.slots, c.total)) {
        s.base = at * c.n_kv;
        s.len = (int)min((int64_t)s.ctx + s.n_nodes, (int64_t)min(s.slots, 0x7fffff00));   // a step beyond it is still a number
    }
    return s;
}

// Bits of 64 neighbouring slots that a node sees, the first of them the slot of node n (n < 0: in the history) and `there` of them
// there.
__device__ __forceinline__ uint64_t tree_seen(const TreeArgs& a, int row, int node, int n, int there)
{
    uint64_t bits;
    n = max(n, -64);
    if (a.mask) {
        const uint64_t* m = a.mask + (int64_t)row * a.words;
        const int w = n >> 6, sh = n & 63;
        if (n == -64) bits = ~0ull;
        else if (n < 0) bits = m[0] << -n | ((1ull << -n) - 1);
        else bits = (w < a.words ? m[w] >> sh : 0) | (sh && w + 1 < a.words ? m[w + 1] << (64 - sh) : 0);
    } else {   // those up to itself
        bits = node - n >= 63 ? ~0ull : node < n ? 0 : (2ull << (node - n)) - 1;
    }
    return there >= 64 ? bits : there > 0 ? bits & ((1ull << there) - 1) : 0;
}

// N neighbouring results of a row's head, e0 on: to its row, or (the engine's projections) to the packed layout.
template <typename T, int N>
__device__ __forceinline__ void tree_store(const TreeArgs& a, int row, int head, int e0, const float (&x)[N])
{
    T r[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (std::is_same<T, _Float16>::value) r[i] = __builtin_bit_cast(_Float16, f2h(x[i]));
        else r[i] = (T)x[i];
    }
    T* to;
    if (a.packed_d) to = (T*)a.out.p + pk_index(row, head * a.c.hd + e0, a.packed_d);
    else to = (T*)a.out.p + (int64_t)row * a.out.row + (int64_t)head * a.out.head + e0;
    typedef uint32_t words __attribute__((ext_vector_type(N * 2 / 4 > 0 ? N * 2 / 4 : 1)));
    if constexpr (N >= 2) *(words*)to = __builtin_bit_cast(words, r);
    else *to = r[0];
}

// Four bytes' codes as halves: two pairs chosen by sel_lo and sel_hi (byte numbers of b:a, zeros between them).
__device__ __forceinline__ uint32_t code_pair(uint32_t a, uint32_t b, uint32_t sel)
{
    const uint32_t u = __builtin_amdgcn_perm(b, a, sel) ^ 0x64806480u;   // 1024 + (code + 128) as halves
    const f16x2 h = __builtin_bit_cast(f16x2, u) - f16x2{(_Float16)1152.f, (_Float16)1152.f};
    return __builtin_bit_cast(uint32_t, h);
}

// sum + a's two values, in fp32.
template <typename T>
__device__ __forceinline__ float add_pair(uint32_t a, float sum)
{
    typedef T t2 __attribute__((ext_vector_type(2)));
    const t2 one = {(T)1.f, (T)1.f};
    if constexpr (std::is_same<T, _Float16>::value) return __builtin_amdgcn_fdot2(__builtin_bit_cast(t2, a), one, sum, false);
    else return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(t2, a), one, sum, false);
}

template <int HD, typename T, typename C, int QT>
__global__ __launch_bounds__(256, QT == 1 ? HD == 64 ? 4 : 3 : 2) void k_attention_tree(TreeArgs a)
{
    typedef typename MathType<C, T>::type M;
    typedef typename Half<M>::x8 m8;
    constexpr bool I8 = std::is_same<C, int8_t>::value;
    constexpr int KS = HD / 32, ET = HD / 16, NW = 4, ROWS = 16 * QT;
    constexpr int ROW = HD * sizeof(C);      // bytes of a vector
    constexpr int KL = ROW / 64;             // 16-byte loads per 16 slots and lane
    constexpr int VW = ET * sizeof(C) / 4;   // words per slot and lane: ET elements
    constexpr bool PAIRS = I8 && std::is_same<T, _Float16>::value && QT == 1;   // weights as sums of two halves
    __shared__ float s_m[NW][ROWS], s_l[NW][ROWS];
    __shared__ int s_odd[NW];
    __shared__ __attribute__((aligned(16))) float s_o[NW][QT][4][64][ET];
    const CacheView& c = a.c;

    // blocks of rows that share their slots are n_kv apart: with 8 heads or a multiple on one die, whose L2 hands the slots on
    const int G = a.heads / c.n_kv, rb = blockIdx.x / c.n_kv, h = blockIdx.x - rb * c.n_kv, chunk = blockIdx.y, j = blockIdx.z;
    const TreeSeq sq = tree_sequence(a, j);
    const int node0 = sq.node0, n_nodes = sq.n_nodes, ctx = sq.ctx, len = sq.len, slots = sq.slots;
    const int n_rows = n_nodes * G, r0 = rb * ROWS;
    const int n_chunks = tree_chunks(len, a.chunk, a.chunks);
    if (r0 >= n_rows || chunk >= n_chunks) return;
    const int s_begin = chunk * a.chunk, s_end = chunk + 1 == n_chunks ? len : s_begin + a.chunk, last = len - 1;
    const int shared_end = min(ctx, len);   // slots before this are seen by every row

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ql = lane & 15, g = lane >> 4;
    const int64_t head_base = sq.base + (int64_t)h * slots;
    const char *K = (const char*)c.k + head_base * ROW, *V = (const char*)c.v + head_base * ROW;
    const float *kscale = I8 ? c.k_scale + head_base : nullptr, *vscale = I8 ? c.v_scale + head_base : nullptr;
    const int first = s_begin + 32 * wave;

    // A step's operands as they come from memory; those of the next step are requested as soon as the registers are free.
    u32x4 kreg[2][KL];
    uint32_t vreg[8][VW];
    f32x4u ks[2], vs[2];
    const unsigned k_off = ql * ROW + 16 * g, v_off = 4 * g * ROW + ET * ql * (int)sizeof(C);
    // rows of one block use the cache's bytes once
    auto load16 = [](const char* p) { return QT == 1 ? __builtin_nontemporal_load((const u32x4*)p) : *(const u32x4*)p; };
    auto load_v = [&](uint32_t (&v)[VW], const char* p) {
        if constexpr (VW == 4) {
            const u32x4 w = load16(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = w[i];
        } else if constexpr (VW == 2) {
            const u32x2 w = QT == 1 ? __builtin_nontemporal_load((const u32x2*)p) : *(const u32x2*)p;
            v[0] = w[0];
            v[1] = w[1];
        } else {
            v[0] = QT == 1 ? __builtin_nontemporal_load((const uint32_t*)p) : *(const uint32_t*)p;
        }
    };
    auto load_keys = [&](int s0) {
        if (s0 + 31 <= last) {
            const char* p = K + (int64_t)s0 * ROW;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < KL; ++i) kreg[kt][i] = load16(p + k_off + kt * 16 * ROW + 64 * i);
            if constexpr (I8)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) ks[kt] = *(const f32x4u*)(kscale + s0 + 4 * g + kt * 16);
        } else {   // slots beyond the last repeat it
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const char* p = K + (int64_t)min(s0 + kt * 16 + ql, last) * ROW + 16 * g;
#pragma unroll
                for (int i = 0; i < KL; ++i) kreg[kt][i] = load16(p + 64 * i);
                if constexpr (I8)
#pragma unroll
                    for (int i = 0; i < 4; ++i) ks[kt][i] = kscale[min(s0 + kt * 16 + 4 * g + i, last)];
            }
        }
    };
    auto load_values = [&](int s0) {
        if (s0 + 31 <= last) {
            const char* p = V + (int64_t)s0 * ROW;
#pragma unroll
            for (int i = 0; i < 8; ++i) load_v(vreg[i], p + v_off + ((i >> 2) * 16 + (i & 3)) * ROW);
            if constexpr (I8)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) vs[kt] = *(const f32x4u*)(vscale + s0 + 4 * g + kt * 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int s = min(s0 + (i >> 2) * 16 + 4 * g + (i & 3), last);
                load_v(vreg[i], V + (int64_t)s * ROW + ET * ql * (int)sizeof(C));
                if constexpr (I8) vs[i >> 2][i & 3] = vscale[s];
            }
        }
    };
    if (first < s_end) {
        load_keys(first);
        load_values(first);
    }

    // queries, and what brings their scores to units of log2: for 16-bit caches a factor sc > 0 (a negative one turns the
    // queries over), else the key's scale times log2_scale, and with bf16 queries the row's power of two in sc
    constexpr bool SCALED = !I8 || !std::is_same<M, T>::value;   // sc is not 1
    const float log2_scale = a.scale * 1.44269504088896341f;
    float sc[QT];
    m8 qf[QT][KS];
    int node[QT];
    u32x4 qreg[QT][KS];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        const int r = min(r0 + u * 16 + ql, n_rows - 1);
        node[u] = r / G;
        const T* qp = (const T*)a.q.p + (int64_t)(node0 + node[u]) * a.q.row + (int64_t)(h * G + r - node[u] * G) * a.q.head;
#pragma unroll
        for (int i = 0; i < KS; ++i) qreg[u][i] = *(const u32x4*)(I8 ? qp + 64 * (i >> 1) + 16 * g + 8 * (i & 1) : qp + 32 * i + 8 * g);
    }
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
    f32x4 o[QT][ET];
    bool odd = false;   // this wave has met a value that is not finite among slots that not every row sees
    float m_run[QT], l_run[QT];
    WeightUnit unit[QT];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
#pragma unroll
        for (int t = 0; t < ET; ++t) o[u][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
        m_run[u] = kLowest;
        l_run[u] = 0.f;
    }
    auto step = [&](int s0, auto tail_step) {
        constexpr bool TAIL = decltype(tail_step)::value;   // some slot is a node's, or there is none
        const int s_next = s0 + 32 * NW;
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
        if (s_next < s_end) load_keys(s_next);
        m8 pb[QT], rest[QT];
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            float mt = kLowest;
            uint32_t seen[2] = {15u, 15u};   // of this lane's slots, by its row
            if constexpr (TAIL) {
                const uint64_t bits = tree_seen(a, node0 + node[u], node[u], s0 - ctx, s_end - s0) >> (4 * g);
                seen[0] = bits & 15;
                seen[1] = bits >> 16 & 15;
            }
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (I8) s[u][kt][i] *= kq[kt][i];
                    if (TAIL && !(seen[kt] >> i & 1)) s[u][kt][i] = -__builtin_inff();
                    mt = fmaxf(mt, s[u][kt][i]);
                }
            mt = across<32>(across<16>(mt, Max()), Max());
            // the weights are relative to a maximum that is followed in steps of 2^8: half holds 2^8 as well as 1
            float alpha = 1.f;
            const bool moves = __any((mt - m_run[u]) * sc[u] > 8.f);
            if (moves) {
                const float m_new = fmaxf(m_run[u], mt);
                alpha = __builtin_amdgcn_exp2f((m_run[u] - m_new) * sc[u]);
                m_run[u] = m_new;
                l_run[u] *= alpha;
                if constexpr (!I8)
#pragma unroll
                    for (int t = 0; t < ET; ++t) o[u][t] *= alpha;
            }
            const float m_sc = I8 ? fmaxf(m_run[u] * sc[u], kLowest) : exponent_top(m_run[u], sc[u], s[u]);   // 8 bits: sc is a power of two
            float top = 0.f;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(SCALED ? fmaf(s[u][kt][i], sc[u], -m_sc) : below_top(s[u][kt][i], m_sc));
                    if constexpr (I8) {
                        l_run[u] += p;
                        s[u][kt][i] = TAIL && !(seen[kt] >> i & 1) ? 0.f : p * vs[kt][i];
                        top = fmaxf(top, fabsf(s[u][kt][i]));
                    } else {
                        pb[u][kt * 4 + i] = (M)p;
                    }
                }
            if constexpr (I8) {
                if (moves || __any(top > unit[u].largest())) {
                    const float f = unit[u].follow(alpha, across<32>(across<16>(top, Max()), Max()));
#pragma unroll
                    for (int t = 0; t < ET; ++t) o[u][t] *= f;
                }
                const float inv = unit[u].inverse();
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        pb[u][kt * 4 + i] = (M)(s[u][kt][i] * inv);
                        if constexpr (PAIRS) rest[u][kt * 4 + i] = (M)fmaf(s[u][kt][i], inv, -(float)pb[u][kt * 4 + i]);
                    }
            }
            if constexpr (!I8)
#pragma unroll
                for (int i = 0; i < 4; ++i) l_run[u] = add_pair<M>(__builtin_bit_cast(u32x4, pb[u])[i], l_run[u]);
        }
        if constexpr (TAIL && !I8) {   // infinite and NaN values count as 0 here, so that no row meets them as 0 * x: see below
            constexpr uint32_t INF = std::is_same<M, _Float16>::value ? 0x7c00u : 0x7f80u;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    const uint32_t x = vreg[i][w], lo = (x & INF) == INF ? 0xffffu : 0u, up = (x >> 16 & INF) == INF ? 0xffff0000u : 0u;
                    odd = odd || (lo | up);
                    vreg[i][w] = x & ~(lo | up);
                }
        }
#pragma unroll
        for (int t = 0; t < ET; ++t) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (I8) w[i] = code_pair(vreg[2 * i][t >> 2], vreg[2 * i + 1][t >> 2], 0x0c040c00u + (t & 3) * 0x00010001u);
                else w[i] = __builtin_amdgcn_perm(vreg[2 * i + 1][t >> 1], vreg[2 * i][t >> 1], t & 1 ? 0x07060302u : 0x05040100u);
            }
            const m8 vf = __builtin_bit_cast(m8, w);
#pragma unroll
            for (int u = 0; u < QT; ++u) {
                o[u][t] = Half<M>::mma(vf, pb[u], o[u][t]);
                if constexpr (PAIRS) o[u][t] = Half<M>::mma(vf, rest[u], o[u][t]);
            }
        }
        if (s_next < s_end) load_values(s_next);
    };
    int s0 = first;
    for (; s0 < s_end && s0 + 31 < shared_end; s0 += 32 * NW) step(s0, std::false_type{});
    for (; s0 < s_end; s0 += 32 * NW) step(s0, std::true_type{});

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
            for (int t = 0; t < ET; t += 4) {
                const float4 x = make_float4(o[u][t][i] * f, o[u][t + 1][i] * f, o[u][t + 2][i] * f, o[u][t + 3][i] * f);
                *(float4*)&s_o[wave][u][i][lane][t] = x;
            }
    }
    __syncthreads();
    // wave i takes elements ET * (4g + i) .. of every row: ET neighbours per lane
    const int e0 = ET * (4 * g + wave);
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        const int r = r0 + u * 16 + ql;
        float x[ET];
#pragma unroll
        for (int t = 0; t < ET; ++t) {
            x[t] = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) x[t] += s_o[w][u][wave][lane][t];
        }
        if (r >= n_rows) continue;
        if constexpr (!I8)
            if (s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3])   // rare: the values that counted as 0, to the rows that see them
                for (int slot = s_begin + max(shared_end - s_begin, 0) / 32 * 32; slot < s_end; ++slot) {
                    if (!tree_seen(a, node0 + node[u], node[u], slot - ctx, 1)) continue;
                    const C* v = (const C*)(V + (int64_t)slot * ROW) + e0;
#pragma unroll
                    for (int t = 0; t < ET; ++t)
                        if (!(fabsf((float)v[t]) <= 3.4e38f)) x[t] += (float)v[t];
                }
        if (n_chunks > 1) {
            float* to = a.part + ((((size_t)j * a.chunks + chunk) * c.n_kv + h) * a.max_nodes * G + r) * (HD + 4);
#pragma unroll
            for (int t = 0; t < ET; t += 4) *(float4*)(to + e0 + t) = make_float4(x[t], x[t + 1], x[t + 2], x[t + 3]);
            if (wave == 0 && g == 0) *(float2*)(to + HD) = make_float2(part_top(m_all[u] * sc[u]), l_all[u]);
        } else {
            const float inv = l_all[u] != 0.f ? 1.f / l_all[u] : 0.f;   // a row that sees nothing gets zeros
#pragma unroll
            for (int t = 0; t < ET; ++t) x[t] *= inv;
            tree_store<T, ET>(a, node0 + r / G, h * G + r % G, e0, x);
        }
    }
}

// Adds up the chunks of rows whose slots were shared out.  A group of HD / 4 lanes adds up chunks like the waves above; WIDE: the groups of
// a workgroup take the chunks of one row in turn (few rows, many chunks: the time is that of the loads one after another), else a
// row each.  15616 rows of few chunks: 5.4 us, with a workgroup a row 17.8; one row of 32 heads at 3900 slots: 3.8 us with WIDE.
template <int HD, typename T, bool WIDE>
__global__ __launch_bounds__(256) void k_tree_join(TreeArgs a)
{
    constexpr int LPG = HD / 4, GROUPS = 256 / LPG;
    __shared__ float s_m[GROUPS], s_l[GROUPS];
    __shared__ float4 s_o[GROUPS][LPG];
    const CacheView& c = a.c;
    const int group = threadIdx.x / LPG, e = threadIdx.x % LPG;
    const int G = a.heads / c.n_kv, per = a.max_nodes * G, h = blockIdx.y, j = blockIdx.z;
    const int r = WIDE ? blockIdx.x : blockIdx.x * GROUPS + group;
    const TreeSeq sq = tree_sequence(a, j);
    const int n = tree_chunks(sq.len, a.chunk, a.chunks);
    if (n < 2 || r >= sq.n_nodes * G) return;
    const size_t step = (size_t)c.n_kv * per * (HD + 4);
    const float* p = a.part + (((size_t)j * a.chunks * c.n_kv + h) * per + r) * (HD + 4);
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
    constexpr int STEP = WIDE ? GROUPS : 1;
    for (int k = WIDE ? group : 0; k < n; k += 4 * STEP) {   // four chunks' loads at a time
        float4 y[4];
        float2 ml[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float* q = p + min(k + i * STEP, n - 1) * step;
            y[i] = *(const float4*)(q + 4 * e);
            ml[i] = *(const float2*)(q + HD);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i * STEP < n) add(ml[i].x, ml[i].y, y[i]);
    }
    if constexpr (WIDE) {
        s_o[group][e] = make_float4(x[0], x[1], x[2], x[3]);
        if (e == 0) {
            s_m[group] = m;
            s_l[group] = l;
        }
        __syncthreads();
        if (group > 0) return;
        for (int k = 1; k < GROUPS; ++k) add(s_m[k], s_l[k], s_o[k][e]);
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= inv;
    tree_store<T, 4>(a, sq.node0 + r / G, h * G + r % G, 4 * e, x);
}

// ------------------------------------------------------------------------------------------ attention of packed prompts
// Causal attention of sequences that lie behind each other: rows offsets[i] .. offsets[i+1] - 1 are sequence i's tokens.  A wave
// takes 32 queries of one head through tiles of 64 keys.  As above the scores are formed as S^T = K Q^T, now in blocks of 32 keys x 32
// queries, so that a query's numbers are in two lanes and the weights are already the operand that O^T += V^T P^T takes:
//   weights  lane (query = lane % 32, hi = lane / 32) holds keys 8b + 4hi + (0..3), b = 0..3, of a block; two b's are an operand
//   values   the same keys of element lane % 32: four neighbouring keys of one element, what the transposed LDS read returns
// Weights are rounded to the values' type, as above, and their sum is that of the rounded ones.
// Keys and values are copied into LDS as they lie in memory (two tiles, one on its way while the other is used), pieces of 16 bytes
// changing places within a row so that what is read at once lies in different banks.
// Bound by power: 12288 tokens, 32 heads on 8 of 128: 1.09 to 1.21 ms by the card, 1.02 to 1.13 PFLOP/s of the half square that counts, where
// zeros take 0.88 (the clock falls to 1.8 GHz, the matrix units are busy 58 % of its cycles).  Several long prompts also by the launch's end,
// their workgroups being of unlike length: six to 4001 tokens 254 us, 0.96 PFLOP/s.  256 prompts to 256 tokens, 32 heads: 215 us, 164 of them bytes.  8 waves a workgroup:
// 1199 -> 1224 and 238 -> 275 us; tiles of 32 keys and 2 waves: 216 -> 237 for the short prompts.
constexpr int kPackTile = 64, kPackQueries = 32;

typedef float f32x16 __attribute__((ext_vector_type(16)));
template <typename T>
__device__ __forceinline__ f32x16 mma32(typename Half<T>::x8 a, typename Half<T>::x8 b, f32x16 c)
{
    if constexpr (std::is_same<T, _Float16>::value) return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef s16x4 __attribute__((address_space(3)))* lds_s16x4;
// 16 lanes: 4 rows x 16 elements; lane i gives the place of elements 4 (i % 4) .. of row i / 4 and gets element i of the rows.
__device__ __forceinline__ uint2 lds_read_transposed(const void* p)
{
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p));
}

template <int HD, typename T, int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_attention_packed(PackedArgs a)
{
    typedef typename Half<T>::x8 t8;
    constexpr int KT = kPackTile, QW = kPackQueries;
    constexpr int ROW = HD * 2, PIECES = ROW / 16;      // bytes and 16-byte pieces of a row
    constexpr int RPC = 64 / PIECES;                    // rows of a copy of 1 KiB
    constexpr int COPIES = KT / RPC / NW;               // copies of a tile per wave
    constexpr int KS = HD / 16, ET = HD / 32;
    constexpr int TILE = KT * ROW;
    static_assert(COPIES * RPC * NW == KT, "whole copies");
    __shared__ __attribute__((aligned(1024))) char lds[2][2][TILE];
    __shared__ int odd_lds;

    // query heads that share a head of keys and values are on one die
    const int G = a.heads / a.n_kv, hk = blockIdx.x % a.n_kv, h = hk * G + blockIdx.x / a.n_kv;
    const int i_seq = blockIdx.y, qt = gridDim.z - 1 - blockIdx.z;
    const int first = a.offsets[i_seq];
    const int end = a.lengths ? first + a.lengths[i_seq] : a.offsets[i_seq + 1];
    const int p = (int)min(table_rows(first, end, INT64_MAX, a.q.rows), (int64_t)a.max_len);
    const int q0 = qt * QW * NW;
    if (q0 >= p) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ql = lane & 31, hi = lane >> 5;
    const int wave_first = q0 + wave * QW, wave_last = wave_first < p ? min(wave_first + QW, p) - 1 : -1;   // -1: no query
    const int n_keys = min(p, q0 + QW * NW), n_tiles = (n_keys + KT - 1) / KT;
    const float sc = fmaxf(fabsf(a.scale) * 1.44269504088896341f, 1e-37f);   // of the scores, in units of log2

    const char* Kg = (const char*)((const T*)a.k.p + (int64_t)first * a.k.row + (int64_t)hk * a.k.head);
    const char* Vg = (const char*)((const T*)a.v.p + (int64_t)first * a.v.row + (int64_t)hk * a.v.head);
    const unsigned k_row = (unsigned)a.k.row * 2, v_row = (unsigned)a.v.row * 2;   // bytes; the host refuses longer rows
    // In 256 bytes, the banks' width, lie the 16-byte pieces of 16 keys' rows that 16 lanes read at once, and the 32 bytes of 4 rows at
    // two places that 32 lanes read transposed.
    auto key_turn = [](int r) { return HD == 128 ? r & 15 : r >> 1 & 7; };
    auto value_turn = [](int r) { return HD == 128 ? (r & 3) << 2 : (r & 2) << 1; };
    // copy c of a wave: rows (c * NW + wave) * RPC + lane / PIECES of the tile; the lane's piece depends on the row's last bits only
    const int c_row = wave * RPC + lane / PIECES;
    const unsigned k_piece = ((lane % PIECES) ^ key_turn(c_row)) * 16, v_piece = ((lane % PIECES) ^ value_turn(c_row)) * 16;
    const unsigned lds_at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)&lds[0][0][0]);
    const unsigned k_off = c_row * k_row + k_piece, v_off = c_row * v_row + v_piece;
    auto copy_tile = [&](int t, int b, bool whole) {
        const char *kp = Kg + (int64_t)t * KT * k_row, *vp = Vg + (int64_t)t * KT * v_row;
        const int left = n_keys - 1 - t * KT;   // last row of the tile that there is; later ones repeat it
#pragma unroll
        for (int c = 0; c < COPIES; ++c) {
            const unsigned place = b * 2 * TILE + (c * NW + wave) * 1024;
            if (whole) {
                lds_copy_1k(lds_at, place, kp + c * NW * RPC * k_row, k_off);
                lds_copy_1k(lds_at, place + TILE, vp + c * NW * RPC * v_row, v_off);
            } else {
                const unsigned r = min(c_row + c * NW * RPC, left);
                lds_copy_1k(lds_at, place, kp, r * k_row + k_piece);
                lds_copy_1k(lds_at, place + TILE, vp, r * v_row + v_piece);
            }
        }
    };
    copy_tile(0, 0, false);
    if (n_tiles > 1) copy_tile(1, 1, false);
    if (threadIdx.x == 0) odd_lds = 0;

    t8 qf[KS];
    const int qpos = min(wave_first + ql, p - 1);
    {
        const T* qp = (const T*)a.q.p + (int64_t)(first + qpos) * a.q.row + (int64_t)h * a.q.head + 8 * hi;
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            u32x4 w = *(const u32x4*)(qp + 16 * ks);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] ^= flip;
            qf[ks] = __builtin_bit_cast(t8, w);
        }
    }
    f32x16 o[ET];
#pragma unroll
    for (int t = 0; t < ET; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m_run = kLowest, l_run = 0.f;

    // places of this lane's pieces: keys' rows are ql (+ 32), values' rows 4hi + (0..3) (+ 8 ...)
    const unsigned k_at = ql * ROW + (hi ^ key_turn(ql)) * 16;   // piece 2 * ks + hi: this with bits of ks turned over
    const int v_r = 4 * hi + ((lane & 15) >> 2);
    unsigned v_at[ET];
#pragma unroll
    for (int t = 0; t < ET; ++t)
        v_at[t] = TILE + v_r * ROW + ((t * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ value_turn(v_r)) * 16 + (lane & 1) * 8;

    // BLOCKS of 32 keys of the tile; DIAGONAL: the last of them is the wave's own, whose key n only queries from n on see
    auto use_tile = [&](auto buffer, int k0, auto blocks, auto diagonal) {
        constexpr int NB = decltype(blocks)::value;
        constexpr bool DIAGONAL = decltype(diagonal)::value;
        const char* tile = &lds[buffer][0][0];
        f32x16 s[NB];
#pragma unroll
        for (int kt = 0; kt < NB; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kt = 0; kt < NB; ++kt) s[kt] = mma32<T>(*(const t8*)(tile + (k_at ^ ks * 32) + kt * 32 * ROW), qf[ks], s[kt]);
        float mt = kLowest;
#pragma unroll
        for (int kt = 0; kt < NB; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (DIAGONAL && kt == NB - 1 && 8 * (i >> 2) + (i & 3) > ql - 4 * hi) s[kt][i] = -__builtin_inff();
                mt = fmaxf(mt, s[kt][i]);
            }
        mt = across<32>(mt, Max());
        // the weights are relative to a maximum that is followed in steps of 2^8: half holds 2^8 as well as 1
        if (__any((mt - m_run) * sc > 8.f)) {
            const float m_new = fmaxf(m_run, mt), alpha = __builtin_amdgcn_exp2f((m_run - m_new) * sc);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int t = 0; t < ET; ++t) o[t] *= alpha;
        }
        const float m_sc = exponent_top(m_run, sc, s);
        t8 pb[2 * NB];
#pragma unroll
        for (int kt = 0; kt < NB; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) pb[kt * 2 + (i >> 3)][i & 7] = (T)__builtin_amdgcn_exp2f(fmaf(s[kt][i], sc, -m_sc));
#pragma unroll
        for (int c = 0; c < 2 * NB; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) l_run = add_pair<T>(__builtin_bit_cast(u32x4, pb[c])[i], l_run);
#pragma unroll
        for (int c = 0; c < 2 * NB; ++c)
#pragma unroll
            for (int t = 0; t < ET; ++t) {
                const uint2 lo = lds_read_transposed(tile + v_at[t] + c * 16 * ROW), up = lds_read_transposed(tile + v_at[t] + (c * 16 + 8) * ROW);
                o[t] = mma32<T>(__builtin_bit_cast(t8, u32x4{lo.x, lo.y, up.x, up.y}), pb[c], o[t]);
            }
    };
    const std::integral_constant<int, 0> even{};
    const std::integral_constant<int, 1> odd{}, one{};
    const std::integral_constant<int, 2> two{};
    // tiles that every query of the workgroup sees whole, an even number of them
    const int n_whole = q0 / KT;
    for (int t = 0; t < n_whole; t += 2) {
        wait_copies_and_meet<0>();   // this tile is there, and nobody reads the other one any more
        if (t) copy_tile(t + 1, 1, true);
        use_tile(even, t * KT, two, std::false_type{});
        wait_copies_and_meet<0>();
        copy_tile(t + 2, 0, t + 2 < n_whole);
        use_tile(odd, t * KT + KT, two, std::false_type{});
    }
    // tiles up to the workgroup's own queries
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    constexpr unsigned short kInf = std::is_same<T, _Float16>::value ? 0x7c00 : 0x7f80;
    for (int t = n_whole; t < n_tiles; ++t) {
        const int k0 = t * KT, buffer = t & 1;
        wait_copies_and_meet<0>();
        if (t && t + 1 < n_tiles) copy_tile(t + 1, (t + 1) & 1, false);
        // infinite and NaN values count as 0 here, so that queries before them do not meet them as 0 * x: see below
        u16x2 top = {0, 0};
        u32x4 w[TILE / 16 / (64 * NW)];
        char* values = &lds[buffer][1][0] + threadIdx.x * 16;
#pragma unroll
        for (int i = 0; i < TILE / 16 / (64 * NW); ++i) {
            w[i] = *(const u32x4*)(values + i * 1024 * NW);
#pragma unroll
            for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w[i][j] & 0x7fff7fffu));
        }
        if (top[0] >= kInf || top[1] >= kInf) {
            for (int i = 0; i < TILE / 16 / (64 * NW) * 8; ++i) {
                uint16_t* x = (uint16_t*)(values + (i >> 3) * 1024 * NW) + (i & 7);
                if ((*x & 0x7fff) >= kInf) *x = 0;
            }
            odd_lds = 1;
        }
        __syncthreads();
        if (k0 > wave_last) continue;
        if (k0 + KT <= wave_first) use_tile(buffer, k0, two, std::false_type{});
        else if (k0 < wave_first) use_tile(buffer, k0, two, std::true_type{});
        else use_tile(buffer, k0, one, std::true_type{});
    }
    // results go through LDS, so that 16 (8) lanes write a head's 256 (128) bytes: a wave has 32 rows of its own there
    const float l = across<32>(l_run, Add()), inv = 1.f / l;
    wait_copies_and_meet<0>();
    char* rows = &lds[0][0][0] + wave * QW * ROW;
    const bool any_odd = odd_lds;
    const float limit = any_odd ? 3.4028235e38f : __builtin_inff();   // half saturates; infinities only below, once they are summed
#pragma unroll
    for (int t = 0; t < ET; ++t)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            T r[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = o[t][4 * b + e] * inv;
                if (std::is_same<T, _Float16>::value && fabsf(x) <= limit) x = fminf(fmaxf(x, -65504.f), 65504.f);   // NaN stays
                r[e] = (T)x;
            }
            *(uint2*)(rows + ql * ROW + (((4 * t + b) ^ key_turn(ql)) * 16 + (hi ^ (ql >> 4)) * 8)) = __builtin_bit_cast(uint2, r);
        }
    if (any_odd)   // rare: the values that counted as 0, to the queries that see them (a positive weight times infinity or NaN)
        for (int e = lane; e < HD; e += 64) {
            float sum = 0.f;
            for (int r = 0, n = q0; r < QW; ++r) {
                for (; n <= min(wave_first + r, wave_last); ++n) {
                    const float x = (float)((const T*)(Vg + (int64_t)n * v_row))[e];
                    if (!(fabsf(x) <= 3.4028235e38f)) sum += x;
                }
                T* to = (T*)(rows + r * ROW + (((e >> 3) ^ key_turn(r)) * 16 + ((e >> 2 & 1) ^ (r >> 4)) * 8)) + (e & 3);
                const float x = (float)*to + sum;
                if constexpr (std::is_same<T, _Float16>::value) *to = __builtin_bit_cast(_Float16, f2h(x));
                else *to = (T)x;
            }
        }
#pragma unroll
    for (int i = 0; i < QW / RPC; ++i) {
        const int r = i * RPC + lane / PIECES, piece = (lane % PIECES) ^ key_turn(r);
        u32x4 w = *(const u32x4*)(rows + r * ROW + (lane % PIECES) * 16);
        if (r >> 4) w = u32x4{w[2], w[3], w[0], w[1]};
        if (wave_first + r >= p) continue;
        const int row = first + wave_first + r;
        T* to = a.packed_d ? (T*)a.out.p + pk_index(row, h * HD + piece * 8, a.packed_d)
                           : (T*)a.out.p + (int64_t)row * a.out.row + (int64_t)h * a.out.head + piece * 8;
        *(u32x4*)to = w;
    }
}

// ------------------------------------------------------------------------------------------ trees of many rows over a cache
// What k_attention_tree computes, for units of more rows than a wave or two can hold: a wave takes 32 rows as the packed kernel takes 32
// queries, the four waves of a workgroup share tiles of 64 slots in LDS, and slots of 8-bit caches become halves once on their way
// there, not once per wave.  Copies of 16-bit slots go straight into LDS; codes pass through registers, requested a tile ahead.
// Bound by vector work and by rows that are not there: 8 trees to 61 nodes at up to 6000 slots, 32 heads on 8, 8 bits, 40 us: 21 vector
// instructions a product, the matrix units 7 % busy; half of the workgroups' rows exist, as a sequence of 3 nodes has as many workgroups as one of 61.
// The kernel above in blocks of 32 rows opens the codes once per block: 75 -> 42 when this one was first measured.
template <int HD, typename T, typename C>
__global__ __launch_bounds__(256, 2) void k_attention_tree_tall(TreeArgs a)
{
    typedef typename MathType<C, T>::type M;
    typedef typename Half<M>::x8 m8;
    constexpr bool I8 = std::is_same<C, int8_t>::value;
    constexpr int NW = 4, KT = 64, QW = 32, ROWS = NW * QW;
    constexpr int ROW = HD * 2, PIECES = ROW / 16, RPC = 64 / PIECES, COPIES = KT / RPC / NW;
    constexpr int KS = HD / 16, ET = HD / 32, TILE = KT * ROW;
    constexpr int PT = HD / 64;   // 16-byte pieces of codes per thread
    __shared__ __attribute__((aligned(1024))) char lds[2][2][TILE];
    __shared__ __attribute__((aligned(16))) float s_ks[2][KT], s_vs[2][KT];
    __shared__ int s_odd;
    const CacheView& c = a.c;
    const int G = a.heads / c.n_kv, rb = blockIdx.x / c.n_kv, h = blockIdx.x - rb * c.n_kv, chunk = blockIdx.y, j = blockIdx.z;
    const TreeSeq sq = tree_sequence(a, j);
    const int node0 = sq.node0, n_nodes = sq.n_nodes, ctx = sq.ctx, len = sq.len;
    const int n_rows = n_nodes * G, r0 = rb * ROWS;
    const int n_chunks = tree_chunks(len, a.chunk, a.chunks);
    if (r0 >= n_rows || chunk >= n_chunks) return;
    const int s_begin = chunk * a.chunk, s_end = chunk + 1 == n_chunks ? len : s_begin + a.chunk, last = len - 1;
    const int shared_end = min(ctx, len);   // slots before this are seen by every row
    const int n_tiles = (s_end - s_begin + KT - 1) / KT;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ql = lane & 31, hi = lane >> 5;
    const int64_t head_base = sq.base + (int64_t)h * sq.slots + s_begin;
    const char *K = (const char*)c.k + head_base * HD * (int)sizeof(C), *V = (const char*)c.v + head_base * HD * (int)sizeof(C);
    const float *kscale = I8 ? c.k_scale + head_base : nullptr, *vscale = I8 ? c.v_scale + head_base : nullptr;
    const int left = last - s_begin;   // last slot there is, from the chunk's first; later ones repeat it

    // banks: see k_attention_packed
    auto key_turn = [](int r) { return HD == 128 ? r & 15 : r >> 1 & 7; };
    auto value_turn = [](int r) { return HD == 128 ? (r & 3) << 2 : (r & 2) << 1; };
    const unsigned lds_at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)&lds[0][0][0]);
    const int c_row = wave * RPC + lane / PIECES;   // 16-bit: row of copy 0
    const unsigned k_piece = ((lane % PIECES) ^ key_turn(c_row)) * 16, v_piece = ((lane % PIECES) ^ value_turn(c_row)) * 16;
    u32x4 kreg[PT], vreg[PT];
    float sreg = 0.f;
    auto request = [&](int t, int b) {
        if constexpr (I8) {
            const int64_t r = min(t * KT + (tid >> 2), left);
#pragma unroll
            for (int i = 0; i < PT; ++i) {
                kreg[i] = *(const u32x4*)(K + r * HD + (i * 4 + (tid & 3)) * 16);
                vreg[i] = *(const u32x4*)(V + r * HD + (i * 4 + (tid & 3)) * 16);
            }
            if (tid < 2 * KT) sreg = (tid < KT ? kscale : vscale)[min(t * KT + (tid & 63), left)];
        } else {
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                const unsigned place = b * 2 * TILE + (i * NW + wave) * 1024, r = min(c_row + i * NW * RPC, left - t * KT);
                lds_copy_1k(lds_at, place, K + (int64_t)t * TILE, r * ROW + k_piece);
                lds_copy_1k(lds_at, place + TILE, V + (int64_t)t * TILE, r * ROW + v_piece);
            }
        }
    };
    const float log2_scale = a.scale * 1.44269504088896341f;
    auto stage = [&](int b) {   // codes to halves
        if constexpr (I8) {
            const int r = tid >> 2;
            auto halves = [](uint32_t lo, uint32_t up) {
                return u32x4{code_pair(lo, lo, 0x0c010c00u), code_pair(lo, lo, 0x0c030c02u), code_pair(up, up, 0x0c010c00u),
                             code_pair(up, up, 0x0c030c02u)};
            };
            // piece 8i + 2 * (tid % 4) + k, turned by its row
            const unsigned to_k = r * ROW + ((2 * (tid & 3)) ^ key_turn(r)) * 16, to_v = r * ROW + ((2 * (tid & 3)) ^ value_turn(r)) * 16;
            char* to = &lds[b][0][0];
#pragma unroll
            for (int i = 0; i < PT; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    *(u32x4*)(to + (to_k ^ (i * 128 + k * 16))) = halves(kreg[i][2 * k], kreg[i][2 * k + 1]);
                    *(u32x4*)(to + TILE + (to_v ^ (i * 128 + k * 16))) = halves(vreg[i][2 * k], vreg[i][2 * k + 1]);
                }
            if (tid < KT) {
                s_ks[b][tid] = sreg * log2_scale;
            } else if (tid < 2 * KT) {
                s_vs[b][tid - KT] = sreg;
            }
        }
    };
    if (n_tiles > 0) request(0, 0);
    if (tid == 0) s_odd = 0;

    // queries and sc: as in k_attention_tree
    constexpr bool SCALED = !I8 || !std::is_same<M, T>::value;
    const int row = min(r0 + wave * QW + ql, n_rows - 1), node = row / G;
    const bool busy = r0 + wave * QW < n_rows;
    float sc = I8 ? 1.f : fmaxf(fabsf(log2_scale), 1e-37f);
    m8 qf[KS];
    {
        const T* qp = (const T*)a.q.p + (int64_t)(node0 + node) * a.q.row + (int64_t)(h * G + row - node * G) * a.q.head + 8 * hi;
        u32x4 w[KS];
#pragma unroll
        for (int i = 0; i < KS; ++i) w[i] = *(const u32x4*)(qp + 16 * i);
        if constexpr (std::is_same<M, T>::value) {
            const uint32_t flip = !I8 && a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
            for (int i = 0; i < KS; ++i) qf[i] = __builtin_bit_cast(m8, w[i] ^ u32x4{flip, flip, flip, flip});
        } else {
            float top = 0.f, x[8];
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                to_floats<T>(w[i], x);
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
            }
            const float down = half_power(across<32>(top, Max()), &sc);
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                to_floats<T>(w[i], x);
#pragma unroll
                for (int e = 0; e < 8; ++e) qf[i][e] = (_Float16)(x[e] * down);
            }
        }
    }
    f32x16 o[ET];
#pragma unroll
    for (int t = 0; t < ET; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m_run = kLowest, l_run = 0.f;
    WeightUnit unit;
    const unsigned k_at = ql * ROW + (hi ^ key_turn(ql)) * 16;
    const int v_r = 4 * hi + ((lane & 15) >> 2);
    unsigned v_at[ET];
#pragma unroll
    for (int t = 0; t < ET; ++t)
        v_at[t] = TILE + v_r * ROW + ((t * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ value_turn(v_r)) * 16 + (lane & 1) * 8;

    auto use_tile = [&](int b, int k0, auto tail_tile) {
        constexpr bool TAIL = decltype(tail_tile)::value;
        const char* tile = &lds[b][0][0];
        f32x16 s[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) s[kt] = mma32<M>(*(const m8*)(tile + (k_at ^ ks * 32) + kt * 32 * ROW), qf[ks], s[kt]);
        if constexpr (I8) __builtin_amdgcn_sched_barrier(0);   // the scales' reads stay behind: their registers are the keys'
        uint64_t seen = ~0ull;
        if constexpr (TAIL) seen = tree_seen(a, node0 + node, node, k0 - ctx, s_end - k0) >> (4 * hi);
        float mt = kLowest;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 kq;
                if constexpr (I8) kq = *(const f32x4*)&s_ks[b][kt * 32 + 8 * g + 4 * hi];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool sees = !TAIL || (seen >> (kt * 32 + 8 * g + e) & 1);
                    float x = s[kt][4 * g + e];
                    if constexpr (I8) x *= kq[e];
                    if (!sees) x = -__builtin_inff();
                    s[kt][4 * g + e] = x;
                    mt = fmaxf(mt, x);
                }
            }
        mt = across<32>(mt, Max());
        float alpha = 1.f;   // see k_attention_tree
        const bool moves = __any((mt - m_run) * sc > 8.f);
        if (moves) {
            const float m_new = fmaxf(m_run, mt);
            alpha = __builtin_amdgcn_exp2f((m_run - m_new) * sc);
            m_run = m_new;
            l_run *= alpha;
            if constexpr (!I8)
#pragma unroll
                for (int t = 0; t < ET; ++t) o[t] *= alpha;
        }
        if constexpr (I8) __builtin_amdgcn_sched_barrier(0);
        const float m_sc = I8 ? fmaxf(m_run * sc, kLowest) : exponent_top(m_run, sc, s);
        m8 pb[4];
        float top = 0.f;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 vq;
                if constexpr (I8) vq = *(const f32x4*)&s_vs[b][kt * 32 + 8 * g + 4 * hi];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = __builtin_amdgcn_exp2f(SCALED ? fmaf(s[kt][4 * g + e], sc, -m_sc) : below_top(s[kt][4 * g + e], m_sc));
                    if constexpr (I8) {
                        l_run += p;
                        s[kt][4 * g + e] = TAIL && !(seen >> (kt * 32 + 8 * g + e) & 1) ? 0.f : p * vq[e];
                        top = fmaxf(top, fabsf(s[kt][4 * g + e]));
                    } else {
                        pb[kt * 2 + (g >> 1)][(g & 1) * 4 + e] = (M)p;
                    }
                }
            }
        if constexpr (I8) {
            if (moves || __any(top > unit.largest())) {
                const float f = unit.follow(alpha, across<32>(top, Max()));
#pragma unroll
                for (int t = 0; t < ET; ++t) o[t] *= f;
            }
            const float inv = unit.inverse();
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) pb[kt * 2 + (i >> 3)][i & 7] = (M)(s[kt][i] * inv);
        }
        if constexpr (!I8)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) l_run = add_pair<M>(__builtin_bit_cast(u32x4, pb[i])[e], l_run);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < ET; ++t) {
                const uint2 lo = lds_read_transposed(tile + v_at[t] + i * 16 * ROW), up = lds_read_transposed(tile + v_at[t] + (i * 16 + 8) * ROW);
                o[t] = mma32<M>(__builtin_bit_cast(m8, u32x4{lo.x, lo.y, up.x, up.y}), pb[i], o[t]);
            }
    };
    // a trip: its tile is in LDS; the next one is requested, codes put into the other half of LDS at its end
    if (n_tiles > 0) stage(0);
    auto trip = [&](int t, auto tail_tile) {
        const int b = t & 1, k0 = s_begin + t * KT;
        wait_copies_and_meet<0>();
        if (t + 1 < n_tiles) request(t + 1, b ^ 1);
        if constexpr (!I8 && decltype(tail_tile)::value) {   // infinite and NaN values count as 0 here, so that no row meets them as 0 * x: see below
            constexpr unsigned short INF = std::is_same<M, _Float16>::value ? 0x7c00 : 0x7f80;
            typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
            u16x2 top = {0, 0};
            char* values = &lds[b][1][0] + tid * 16;
#pragma unroll
            for (int i = 0; i < TILE / 4096; ++i) {
                const u32x4 w = *(const u32x4*)(values + i * 4096);
#pragma unroll
                for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w[e] & 0x7fff7fffu));
            }
            if (top[0] >= INF || top[1] >= INF) {
                for (int i = 0; i < TILE / 4096 * 8; ++i) {
                    uint16_t* x = (uint16_t*)(values + (i >> 3) * 4096) + (i & 7);
                    if ((*x & 0x7fff) >= INF) *x = 0;
                }
                s_odd = 1;
            }
            __syncthreads();
        }
        if (busy) use_tile(b, k0, tail_tile);
        if (I8 && t + 1 < n_tiles) stage(b ^ 1);   // last read before this trip's barrier
    };
    const int n_shared = min(n_tiles, max(shared_end - s_begin, 0) / KT);   // tiles that every row sees whole
    for (int t = 0; t < n_shared; ++t) trip(t, std::false_type{});
    for (int t = n_shared; t < n_tiles; ++t) trip(t, std::true_type{});
    const float l = across<32>(l_run, Add());
    wait_copies_and_meet<0>();
    if (r0 + wave * QW + ql >= n_rows) return;
    const float f = (I8 ? unit.R : 1.f) * (n_chunks > 1 ? 1.f : l != 0.f ? 1.f / l : 0.f);   // a row that sees nothing gets zeros
    float* const part = a.part + ((((size_t)j * a.chunks + chunk) * c.n_kv + h) * a.max_nodes * G + row) * (HD + 4);
    if (n_chunks > 1 && hi == 0) *(float2*)(part + HD) = make_float2(part_top(m_run * sc), l);
#pragma unroll
    for (int t = 0; t < ET; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e0 = 32 * t + 8 * i + 4 * hi;
            float x[4] = {o[t][4 * i] * f, o[t][4 * i + 1] * f, o[t][4 * i + 2] * f, o[t][4 * i + 3] * f};
            if constexpr (!I8)
                if (s_odd)   // rare: the values that counted as 0, to the rows that see them (a positive weight times infinity or NaN)
                    for (int slot = s_begin + max(shared_end - s_begin, 0) / KT * KT; slot < s_end; ++slot)
                        if (tree_seen(a, node0 + node, node, slot - ctx, 1))
                            for (int e = 0; e < 4; ++e) {
                                const float y = (float)((const C*)V)[(int64_t)(slot - s_begin) * HD + e0 + e];
                                if (!(fabsf(y) <= 3.4e38f)) x[e] += y;
                            }
            if (n_chunks > 1) *(float4*)(part + e0) = make_float4(x[0], x[1], x[2], x[3]);
            else tree_store<T, 4>(a, node0 + node, h * G + row - node * G, e0, x);
        }
}

// ------------------------------------------------------------------------------------------ launches
template <int HD, typename TOKEN, typename CACHE>
static void cache_write(const CacheView& c, const RowsView& k, const RowsView& v, const int32_t* seq, const int32_t* slot, int n, hipStream_t s)
{
    constexpr int heads = kCachePasses * CachePlace::step(HD);
    k_cache_write<HD, TOKEN, CACHE><<<dim3((n + kCacheTokens - 1) / kCacheTokens, (c.n_kv + heads - 1) / heads, 2), 256, 0, s>>>(c, k, v, seq, slot, n);
}
template <int HD, typename TOKEN, typename CACHE>
static void cache_read(const CacheView& c, const RowsView& k, const RowsView& v, const int32_t* seq, const int32_t* slot, int n, hipStream_t s)
{
    constexpr int heads = kCachePasses * CachePlace::step(HD);
    k_cache_read<HD, TOKEN, CACHE><<<dim3((n + kCacheTokens - 1) / kCacheTokens, (c.n_kv + heads - 1) / heads, 2), 256, 0, s>>>(c, k, v, seq, slot, n);
}
// f(head dim, tokens' type, cache's type) with values of those types and dims.
template <class F>
static void with_types(int hd, int token, int cache, F f)
{
    auto by_cache = [&](auto dim, auto t) {
        if (cache == kI8) f(dim, t, int8_t{});
        else if (cache == kF16) f(dim, t, _Float16{});
        else f(dim, t, __bf16{});
    };
    auto by_token = [&](auto dim) {
        if (token == kF16) by_cache(dim, _Float16{});
        else by_cache(dim, __bf16{});
    };
    if (hd == 128) by_token(std::integral_constant<int, 128>{});
    else by_token(std::integral_constant<int, 64>{});
}

void launch_cache_write(const CacheView& c, const RowsView& k, const RowsView& v, int token, const int32_t* seq, const int32_t* slot, int n,
                        hipStream_t s)
{
    with_types(c.hd, token, c.dtype, [&](auto dim, auto t, auto e) { cache_write<decltype(dim)::value, decltype(t), decltype(e)>(c, k, v, seq, slot, n, s); });
}

void launch_cache_read(const CacheView& c, const RowsView& k, const RowsView& v, int token, const int32_t* seq, const int32_t* slot, int n,
                       hipStream_t s)
{
    with_types(c.hd, token, c.dtype, [&](auto dim, auto t, auto e) { cache_read<decltype(dim)::value, decltype(t), decltype(e)>(c, k, v, seq, slot, n, s); });
}

void launch_rotate_store(const MbState& st, const float* qkv_part, int ksplit, size_t part_stride, const float* rope_cos, const float* rope_sin,
                         f16_t* rows, int dense_kv, const CacheView& c, const int32_t* slot, int d, int n_max, hipStream_t s)
{
    auto go = [&](auto dim, auto t) {
        constexpr int HD = decltype(dim)::value;
        const dim3 grid(n_max, (3 * c.n_kv * HD + 2047) / 2048);
        k_rotate_store<HD, decltype(t)><<<grid, 256, 0, s>>>(st, qkv_part, ksplit, part_stride, rope_cos, rope_sin, rows, dense_kv, c, slot, d);
    };
    auto by_cache = [&](auto dim) {
        if (c.dtype == kI8) go(dim, int8_t{});
        else go(dim, _Float16{});
    };
    if (c.hd == 128) by_cache(std::integral_constant<int, 128>{});
    else by_cache(std::integral_constant<int, 64>{});
}

template <int HD, typename T, typename C>
static void attention_tree(const TreeArgs& a, int tiles, hipStream_t s)
{
    const dim3 grid(a.c.n_kv * a.row_blocks, a.chunks, a.n_seq);
    if (tiles == 1) k_attention_tree<HD, T, C, 1><<<grid, 256, 0, s>>>(a);
    else if (tiles == 2) k_attention_tree<HD, T, C, 2><<<grid, 256, 0, s>>>(a);
    else k_attention_tree_tall<HD, T, C><<<grid, 256, 0, s>>>(a);
    if (a.chunks < 2) return;
    // A row's chunks one after another are slower than a workgroup's start where there are more than a few and the rows leave units idle.
    // Whole calls, us, a workgroup a row / a group of lanes a row: 32 rows of 9 chunks 13.4 / 14.2, of 16 14.3 / 16.0, of 24 48.7 / 51.8, of 92
    // 82.1 / 91.9; 512 rows of 24 54.5 / 57.7; 1024 of 11 35.9 / 34.9 and 58.6 / 58.8, 2048 99.0 / 98.1; beyond 4096 the other way: 8192 327.2 / 321.6,
    // 15616 of 12 56.9 / 46.0.
    const int rows = a.max_nodes * (a.heads / a.c.n_kv), groups = 1024 / HD;
    if (a.chunks > 8 && (int64_t)rows * a.c.n_kv * a.n_seq <= 4096) k_tree_join<HD, T, true><<<dim3(rows, a.c.n_kv, a.n_seq), 256, 0, s>>>(a);
    else k_tree_join<HD, T, false><<<dim3((rows + groups - 1) / groups, a.c.n_kv, a.n_seq), 256, 0, s>>>(a);
}

void launch_attention_tree(const TreeArgs& a, int token, int tiles, hipStream_t s)
{
    with_types(a.c.hd, token, a.c.dtype, [&](auto dim, auto t, auto e) {
        typedef decltype(t) T;
        typedef decltype(e) C;
        if constexpr (std::is_same<C, int8_t>::value || std::is_same<C, T>::value) {
            attention_tree<decltype(dim)::value, T, C>(a, tiles, s);
        }
    });
}

template <int HD, typename T>
static void attention_packed(const PackedArgs& a, int n_seq, hipStream_t s)
{
    constexpr int NW = 4, QUERIES = kPackQueries * NW;
    k_attention_packed<HD, T, NW><<<dim3(a.heads, n_seq, (a.max_len + QUERIES - 1) / QUERIES), 64 * NW, 0, s>>>(a);
}

void launch_attention_packed(const PackedArgs& a, int hd, int token, int n_seq, hipStream_t s)
{
    if (hd == 128) token == kF16 ? attention_packed<128, _Float16>(a, n_seq, s) : attention_packed<128, __bf16>(a, n_seq, s);
    else token == kF16 ? attention_packed<64, _Float16>(a, n_seq, s) : attention_packed<64, __bf16>(a, n_seq, s);
}

}  // namespace ss

#endif

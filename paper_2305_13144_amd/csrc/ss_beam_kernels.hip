// Kernels of beam search: of all continuations of a group's beams the best ones.
#include <cfloat>
#include <climits>
#include <type_traits>

#include "ss_device.h"
#include "ss_plan.h"

namespace ss {

// Two launches.  k_beam_rows takes a row's logits once, in `slices` workgroups: the sum of their exponentials, and the `keep` best candidates (of one
// beam no more can be taken).  k_beam_pick joins a group's: the rows' log sums and all ranks in float64, and their order.
constexpr float kLog2e = 1.44269504088896341f;

// 16 bytes of logits as floats.
template <typename T>
struct LogitVector;
template <>
struct LogitVector<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void open(const u32x4& r, float (&v)[N])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __uint_as_float(r[i]);
    }
};
template <>
struct LogitVector<_Float16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void open(const u32x4& r, float (&v)[N])
    {
        const f16x8 h = __builtin_bit_cast(f16x8, r);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (float)h[i];
    }
};
template <>
struct LogitVector<__bf16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void open(const u32x4& r, float (&v)[N])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(r[i] << 16);
            v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
        }
    }
};

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

// A number's bits, ordered as the numbers; -0, which is equal to +0, becomes it.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A number that at least n of four values of each lane are not below: the n-th largest but for its last 16 bits, bit by bit; -inf where that is -inf.
__device__ __forceinline__ float nth_largest(const f32x4& x, int n)
{
    uint32_t t = 0;
    for (int b = 31; b >= 16; --b) {
        int there = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) there += __popcll(__ballot(ordered(x[i]) >= (t | 1u << b)));
        if (there >= n) t |= 1u << b;
    }
    const float least = __uint_as_float(t & 0x80000000u ? t & 0x7fffffffu : ~t);
    return least >= -3.4028235e38f ? least : -__builtin_inff();   // -inf without its last bits is a NaN
}

// The candidates that a wave has met and not ruled out, in no order, in LDS.
struct Shortlist {
    float* v;
    int* i;   // tokens
    int count;

    // Only the n best stay (larger logits, of equal ones lower tokens), where there are more; returns the n-th's logit.
    __device__ __forceinline__ float cut(int n)
    {
        const int lane = threadIdx.x & 63, rounds = (count + 63) >> 6;
        auto held = [&](int r) { return r * 64 + lane < count ? ordered(v[r * 64 + lane]) : 0u; };   // 0: none, below all
        auto at_least = [&](auto f) {
            int there = 0;
            for (int r = 0; r < rounds; ++r) there += __popcll(__ballot(f(r)));
            return there;
        };
        uint32_t t = 0;
        for (int b = 31; b >= 0; --b)
            if (at_least([&](int r) { return held(r) >= (t | 1u << b); }) >= n) t |= 1u << b;
        // of those that are equal to it the first ones: tokens below `to`
        const int equal = n - at_least([&](int r) { return held(r) > t; });
        int to = INT_MAX;
        if (at_least([&](int r) { return held(r) == t; }) > equal) {
            to = 0;
            for (int b = 30; b >= 0; --b)   // the largest number that no more than `equal` tokens are below
                if (at_least([&](int r) { return held(r) == t && i[r * 64 + lane] < (to | 1 << b); }) <= equal) to |= 1 << b;
        }
        int kept = 0;
        for (int r = 0; r < rounds; ++r) {   // what is written is what has been read
            const uint32_t h = held(r);
            const int token = h ? i[r * 64 + lane] : 0;
            const bool stays = h > t || (h == t && token < to);
            const uint64_t all = __ballot(stays);
            const float x = h ? v[r * 64 + lane] : 0.f;
            if (stays) {
                const int at = kept + __popcll(all & ((1ull << lane) - 1));
                v[at] = x;
                i[at] = token;
            }
            kept += __popcll(all);
        }
        count = kept;
        return __uint_as_float(t & 0x80000000u ? t & 0x7fffffffu : ~t);
    }
};

// A wave goes through its part of a row in order, 64 x 16 bytes a step, kBeamAhead steps requested at a time.
//   sum         of exp(x - ref): ref is the largest logit so far (first of kBeamAhead steps).  It moves a few times in a row without an order, at each step of one
//               that ascends (768 rows of 100003 fp32 logits 219 us, 204 where it moved from 80 above it on, which cost the largest terms 2^-18 by
//               their exponents' rounding).  Exponents are off by 2.25 * 2^-24 of themselves, which is 2.25 * 2^-24 (max - mean logit) of the sum, the mean by
//               the probabilities; no row's is further than log(vocab) from the maximum.  Exponentials are off by 2^-23; those of 16 bytes are added
//               in fp32, and their sums in fp64, as thousands of terms follow each other: 5 * 2^-24 more.  The largest logit's is 1, the log of the sum not below 0
//   candidates  a lane keeps the largest of its 16 bytes' largest logits, with its step, and the second largest: 4 instructions a step, whatever
//               the order of the logits.  The keep-th largest of the workgroup's lanes, `least`, is what none of the keep best is below; so those are
//               in the 16 bytes that a lane remembers, read again, and where a lane's second is not below it either, in the whole of what
//               that lane has read (some 1 in 30 waves).  Where that is so in many lanes, as with few distinct logits, the wave goes through all of
//               its part again
// NaN and +inf, which are no candidates, would show in the sum: then the wave goes through its part once more and takes them as -inf.
// Bound by the bytes and, at 16 bits, by the vector units (about 9 instructions a logit, 4 of them the exponential's).  Lists in order of the lanes of a
// wave, into which every logit above the last went by itself, took 17 of 57 us (96 x 8 rows over 100003 tokens), one that grew to 64 and
// was then cut to its best 35 of 78.
constexpr int kBeamAhead = 4, kBeamList = 64, kBeamLanes = 6;

template <typename T>
__global__ __launch_bounds__(256) void k_beam_rows(BeamArgs a)
{
    typedef LogitVector<T> Vec;
    constexpr int N = Vec::N, NW = 4, CAP = kBeamList + 64 * N;
    __shared__ float s_v[NW * CAP], s_ref[NW];
    __shared__ int s_i[NW * CAP], s_count[NW];
    __shared__ double s_sum[NW];
    __shared__ __attribute__((aligned(16))) float s_first[256];
    const int row = blockIdx.y, slice = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    if (a.ended && a.ended[row]) return;
    const T* x = (const T*)a.logits + (int64_t)row * a.row_stride;
    const int mis = (int)((uintptr_t)x & 15) / (int)sizeof(T);   // elements of the first 16 bytes that are before the row
    const int64_t steps_all = ((int64_t)mis + a.vocab + 64 * N - 1) / (64 * N), workers = (int64_t)a.slices * NW, me = (int64_t)slice * NW + wave;
    const int first = (int)(steps_all * me / workers), end = (int)(steps_all * (me + 1) / workers);

    // 16 bytes: those of a lane in a step; at the row's ends element by element, -inf beside it
    auto place = [&](int s, int l) { return (int64_t)s * (64 * N) - mis + l * N; };
    auto load_one = [&](int64_t e, u32x4& r) {
        if (e >= 0 && e + N <= a.vocab) {
            r = *(const u32x4*)(x + e);
            return;
        }
        T part[N];
#pragma unroll
        for (int i = 0; i < N; ++i) part[i] = e + i >= 0 && e + i < a.vocab ? x[e + i] : (T)(-__builtin_inff());
        r = __builtin_bit_cast(u32x4, part);
    };
    auto load = [&](int s, u32x4& r) {
        if (place(s, 0) >= 0 && place(s, 64) <= a.vocab) r = __builtin_nontemporal_load((const u32x4*)(x + place(s, lane)));
        else load_one(place(s, lane), r);
    };
    auto clean = [&](float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] <= 3.4028235e38f ? v[i] : -__builtin_inff();
    };
    auto largest = [&](const float (&v)[N]) {
        float m = v[0];
#pragma unroll
        for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
        return m;
    };

    float ref, best, second;   // of this lane's 16 bytes, by their largest logits
    int best_step;
    double sum;
    auto pass = [&](auto clean_pass) {
        constexpr bool CLEAN = decltype(clean_pass)::value;
        auto open = [&](const u32x4& r, float (&v)[N]) {
            Vec::open(r, v);
            if constexpr (CLEAN) clean(v);
        };
        u32x4 now[kBeamAhead], next[kBeamAhead];
#pragma unroll
        for (int k = 0; k < kBeamAhead; ++k) {
            next[k] = u32x4{0, 0, 0, 0};
            if (first + k < end) load(first + k, next[k]);
        }
        ref = -3.4028235e38f;   // the lowest: a row may hold nothing else
#pragma unroll
        for (int k = 0; k < kBeamAhead; ++k)
            if (first + k < end) {
                float v[N];
                open(next[k], v);
                ref = fmaxf(ref, largest(v));
            }
        ref = wave_max(ref);
        best = second = -__builtin_inff();
        best_step = first;
        sum = 0;
        for (int s = first; s < end; s += kBeamAhead) {
#pragma unroll
            for (int k = 0; k < kBeamAhead; ++k) now[k] = next[k];
#pragma unroll
            for (int k = 0; k < kBeamAhead; ++k)
                if (s + kBeamAhead + k < end) load(s + kBeamAhead + k, next[k]);
#pragma unroll
            for (int k = 0; k < kBeamAhead; ++k) {
                if (s + k >= end) break;
                float v[N];
                open(now[k], v);
                const float top = largest(v);
                if (__any(top > ref)) {
                    const float moved = wave_max(top);
                    sum *= exp((double)ref - (double)moved);
                    ref = moved;
                }
                float p[N];
#pragma unroll
                for (int i = 0; i < N; ++i) p[i] = __builtin_amdgcn_exp2f((v[i] - ref) * kLog2e);
#pragma unroll
                for (int w = N / 2; w > 0; w >>= 1)
#pragma unroll
                    for (int i = 0; i < w; ++i) p[i] += p[i + w];
                sum += (double)p[0];
                second = fmaxf(second, fminf(best, top));
                best_step = top > best ? s + k : best_step;
                best = fmaxf(best, top);
            }
        }
        sum = wave_sum(sum);
        return fabs(sum) <= 1e300;
    };
    if (!pass(std::false_type{})) pass(std::true_type{});
    s_first[t] = best;
    __syncthreads();
    const float least = nth_largest(*(const f32x4*)(s_first + 4 * lane), a.keep);

    Shortlist list{s_v + wave * CAP, s_i + wave * CAP, 0};
    auto collect = [&](bool have, const u32x4& r, int64_t e, float above) {   // of a lane's 16 bytes at e; cut: only the best stay, and the last's logit
        float v[N];
        Vec::open(r, v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool goes = have && v[i] >= least && v[i] > above && v[i] <= 3.4028235e38f;
            const uint64_t all = __ballot(goes);
            if (goes) {
                const int at = list.count + __popcll(all & ((1ull << lane) - 1));
                list.v[at] = v[i];
                list.i[at] = (int)(e + i);
            }
            list.count += __popcll(all);
        }
        return list.count > kBeamList ? list.cut(a.keep) : -__builtin_inff();
    };
    constexpr float kNothing = -__builtin_inff();
    const bool here = best >= least && best > kNothing;
    uint64_t more = __ballot(here && second >= least && second > kNothing);
    if (__popcll(more) <= kBeamLanes) {
        u32x4 r{0, 0, 0, 0};
        const int64_t e = place(best_step, lane);
        if (here) load_one(e, r);
        if (__any(here)) collect(here, r, e, kNothing);
        for (; more; more &= more - 1) {
            const int l = __ffsll((unsigned long long)more) - 1, known = __builtin_amdgcn_readlane(best_step, l);
            for (int s0 = first; s0 < end; s0 += 64) {
                const int s = s0 + lane;
                const int64_t at = place(s, l);
                const bool have = s < end && s != known;
                if (have) load_one(at, r);
                collect(have, r, at, kNothing);
            }
        }
    } else {
        float above = kNothing;   // once the list has been cut: `keep` of its candidates, all before those to come, are not below it
        for (int s = first; s < end; ++s) {
            u32x4 r;
            load(s, r);
            above = fmaxf(above, collect(true, r, place(s, lane), above));
        }
    }

    // the waves' together
    if (lane == 0) {
        s_count[wave] = list.count;
        s_ref[wave] = ref;
        s_sum[wave] = sum;
    }
    __syncthreads();
    float* out = a.part + ((int64_t)row * a.slices + slice) * beam_part_floats(a.keep);
    if (t == 0) {
        float top = s_ref[0];
        for (int w = 1; w < NW; ++w) top = fmaxf(top, s_ref[w]);
        double all = 0;
        for (int w = 0; w < NW; ++w) all += s_sum[w] * exp((double)s_ref[w] - (double)top);
        out[0] = top;
        *(double*)(out + 2) = all;
    }
    int n = 0;
    for (int w = 0; w < NW; ++w) n += s_count[w];
    if (lane < s_count[wave]) {   // at most kBeamList of a wave
        const float v = list.v[lane];
        const int i = list.i[lane];
        int before = 0;
        for (int w = 0; w < NW; ++w) {
            const int there = s_count[w];
#pragma unroll 8
            for (int k = 0; k < there; ++k) before += (s_v[w * CAP + k] > v) | ((s_v[w * CAP + k] == v) & (s_i[w * CAP + k] < i));
        }
        if (before < a.keep) {
            out[4 + before] = v;
            out[4 + a.keep + before] = __int_as_float(i);
        }
    }
    if (t >= n && t < a.keep) out[4 + a.keep + t] = __int_as_float(-1);   // fewer candidates than places
}

// Tokens of a beam of this length, and with one more.
__device__ __forceinline__ int beam_length(int length, bool more) { return min(max(length, 0), INT_MAX - more) + more; }

// Up to kBeamRanked candidates find their places by counting those before them, once each wave has left out what is not among its best; more (then a row is one slice) are taken one by one, a lane of
// the first wave holding the best of its beam that is left.  Bound by a chain of latencies (a launch's start, two loads behind each other, fp64 exp,
// log and pow of a lane per beam): all that does not depend on other loads is requested at the start.  512 threads, two candidates each, against 256 of four: 6.2 for 6.9 us
// (4 beams, 32000 logits), 7.6 for 8.9 (32 x 8), 7.2 for 9.4 (96 x 8, 100003 logits).
constexpr int kPickThreads = 512;
__global__ __launch_bounds__(kPickThreads) void k_beam_pick(BeamArgs a)
{
    struct Ranked {
        double rank;
        uint64_t key;   // beam and token: of equal ranks the lower one is first
    };
    constexpr uint64_t kNone = ~0ull;
    constexpr int NT = kPickThreads, NW = NT / 64, PER = kBeamRanked / NT;
    __shared__ Ranked s_c[kBeamRanked];
    __shared__ double s_top[kBeamMax], s_log[kBeamMax], s_total[kBeamMax], s_power[kBeamMax];
    __shared__ int s_over[kBeamMax], s_row[kBeamMax], s_token[kBeamMax], s_len[kBeamMax], s_kept[NW];
    const int g = blockIdx.x, t = threadIdx.x, per = beam_part_floats(a.keep), lists = a.slices * a.keep, n = a.beams * lists, sums = a.beams * a.slices;
    const float* part = a.part + (int64_t)g * a.beams * a.slices * per;
    const bool ranked = n <= kBeamRanked;
    // (sums <= n: with one slice a row there are at most kBeamMax of them)
    float ref[PER], cand[PER];
    double sum_of[PER];
    int token_of[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = t + NT * k;
        if (c < sums) {
            ref[k] = part[c * per];
            sum_of[k] = *(const double*)(part + c * per + 2);
        }
        if (ranked && c < n) {
            const float* p = part + (int64_t)(c / a.keep) * per + 4 + c % a.keep;
            cand[k] = *p;
            token_of[k] = __float_as_int(p[a.keep]);
        }
    }
    if (t < a.beams) {
        const int row = g * a.beams + t, len = a.lengths ? a.lengths[row] : 0;
        const bool over = a.ended && a.ended[row];
        s_over[t] = over;
        s_len[t] = len;
        s_total[t] = a.totals[row];
        const double scale = a.power != 0.f ? pow((double)max(beam_length(len, !over), 1), (double)a.power) : 1.0;
        s_power[t] = scale > 0 ? scale : DBL_MIN;   // where a power is below all numbers a sum of 0 still has the rank 0
    }
    if (t < a.keep) s_row[t] = s_token[t] = -1;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = t + NT * k;
        if (c < sums) s_c[c].rank = ref[k];
    }
    __syncthreads();
    double share[PER];   // a slice's sum, relative to its row's largest reference
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = t + NT * k;
        if (c >= sums) break;
        const int beam = c / a.slices;
        if (s_over[beam]) continue;
        double m = s_c[beam * a.slices].rank;
        for (int o = 1; o < a.slices; ++o) m = fmax(m, s_c[beam * a.slices + o].rank);
        share[k] = sum_of[k] * exp((double)ref[k] - m);
        s_top[beam] = m;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = t + NT * k;
        if (c < sums) s_c[c].rank = share[k];
    }
    __syncthreads();
    if (t < a.beams && !s_over[t]) {
        double l = s_c[t * a.slices].rank;
        for (int o = 1; o < a.slices; ++o) l += s_c[t * a.slices + o].rank;
        s_log[t] = log(l);
    }
    __syncthreads();
    // a candidate of a beam, its e-th: its rank and its sum
    auto candidate = [&](int beam, int e, float logit, int token, double* sum, uint64_t* key) {
        *key = kNone;
        *sum = -__builtin_inf();
        if (!(fabs(s_total[beam]) <= 3.5e38)) return -__builtin_inf();
        if (s_over[beam]) {
            if (e > 0) return -__builtin_inf();
            *sum = s_total[beam];
            *key = (uint64_t)beam << 32 | (uint32_t)max(a.end_id, 0);
        } else {
            if (token < 0) return -__builtin_inf();
            *sum = s_total[beam] + (((double)logit - s_top[beam]) - s_log[beam]);
            *key = (uint64_t)beam << 32 | (uint32_t)token;
        }
        return *sum / s_power[beam];
    };
    auto take = [&](int place, uint64_t key, double sum) {
        const int beam = (int)(key >> 32), row = g * a.beams + beam, at = g * a.keep + place;
        const bool over = s_over[beam];
        const int token = over ? a.end_id : (int)(uint32_t)key;
        s_row[place] = row;
        s_token[place] = over ? -1 : token;   // to be appended
        a.parent[at] = row;
        a.token[at] = token;
        a.next_totals[at] = (float)sum;
        if (a.next_lengths) a.next_lengths[at] = beam_length(s_len[beam], !over);
        if (a.next_ended) a.next_ended[at] = over || token == a.end_id;
    };
    if (ranked) {
        // of each wave's candidates those that are not below its keep-th, as floats, which are ordered alike
        Ranked mine[PER];
        double sum[PER];
        uint32_t as_float[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int c = t + NT * k;
            mine[k] = {-__builtin_inf(), kNone};
            if (c < n) mine[k].rank = candidate(c / lists, c % lists, cand[k], token_of[k], &sum[k], &mine[k].key);
            as_float[k] = ordered((float)mine[k].rank);
        }
        uint32_t least = 0;   // but for its last bits
        for (int b = 31; b >= 12; --b) {
            int there = 0;
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (NT * k < n) there += __popcll(__ballot(as_float[k] >= (least | 1u << b)));
            if (there >= a.keep) least |= 1u << b;
        }
        int kept = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (NT * k >= n) break;
            const bool stays = mine[k].key != kNone && as_float[k] >= least;
            const uint64_t all = __ballot(stays);
            if (stays) s_c[(t >> 6) * (64 * PER) + kept + __popcll(all & ((1ull << (t & 63)) - 1))] = mine[k];
            else mine[k].key = kNone;
            kept += __popcll(all);
        }
        if ((t & 63) == 0) s_kept[t >> 6] = kept;
        __syncthreads();
        int before[PER] = {};
        for (int w = 0; w < NW; ++w) {
            const int there = s_kept[w];
#pragma unroll 4
            for (int o = 0; o < there; ++o) {
                const Ranked x = s_c[w * (64 * PER) + o];
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (NT * k < n) before[k] += (x.rank > mine[k].rank) | ((x.rank == mine[k].rank) & (x.key < mine[k].key));
            }
        }
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (mine[k].key != kNone && before[k] < a.keep) take(before[k], mine[k].key, sum[k]);
    } else if (t < 64) {
        int at = 0;
        double sum = 0, rank = -__builtin_inf();
        uint64_t key = kNone;
        auto head = [&] {
            const float* p = part + (int64_t)t * per + 4 + at;
            rank = candidate(t, at, *p, __float_as_int(p[a.keep]), &sum, &key);
        };
        if (t < a.beams) head();
        for (int place = 0; place < a.keep; ++place) {
            double r = rank;
            uint64_t best = key;
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) {
                const double o = __shfl_xor(r, d);
                const uint64_t ok = __shfl_xor((unsigned long long)best, d);
                if (o > r || (o == r && ok < best)) {
                    r = o;
                    best = ok;
                }
            }
            if (best == kNone) break;
            if (key == best) {
                take(place, key, sum);
                if (++at < a.keep) head();
                else {
                    rank = -__builtin_inf();
                    key = kNone;
                }
            }
        }
    }
    __syncthreads();
    if (t < a.keep && s_row[t] < 0) {   // fewer candidates than places
        const int at = g * a.keep + t;
        a.parent[at] = a.token[at] = -1;
        a.next_totals[at] = -__builtin_inff();
        if (a.next_lengths) a.next_lengths[at] = 0;
        if (a.next_ended) a.next_ended[at] = 1;
    }
    if (!a.next_history) return;
    constexpr int AT_ONCE = 16;   // a wave takes a history, so many loads at a time
    const int width = a.next_history_stride;
    for (int k = t >> 6; k < a.keep; k += NW) {
        const int row = s_row[k], len = row < 0 ? 0 : max(s_len[row - g * a.beams], 0), token = s_token[k], kept = min(len, a.history_stride);
        const int32_t* from = a.history + (int64_t)max(row, 0) * a.history_stride;
        int32_t* to = a.next_history + ((int64_t)g * a.keep + k) * width;
        for (int i0 = t & 63; i0 < width; i0 += 64 * AT_ONCE) {
            int x[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int i = i0 + 64 * u;
                x[u] = i == len ? token : -1;
                if (i < kept) x[u] = from[i];
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (i0 + 64 * u < width) to[i0 + 64 * u] = x[u];
        }
    }
}

void launch_beam_select(const BeamArgs& a, int dtype, hipStream_t s)
{
    const dim3 grid(a.slices, a.n_groups * a.beams);
    if (dtype == kF32) k_beam_rows<float><<<grid, 256, 0, s>>>(a);
    else if (dtype == kF16) k_beam_rows<_Float16><<<grid, 256, 0, s>>>(a);
    else k_beam_rows<__bf16><<<grid, 256, 0, s>>>(a);
    k_beam_pick<<<a.n_groups, kPickThreads, 0, s>>>(a);
}

}  // namespace ss

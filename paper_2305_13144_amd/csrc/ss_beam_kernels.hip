// Kernels of beam search: of all continuations of a group's beams the best ones.
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

// The best candidates that a wave has met, lane k the k-th: larger logits first, of equal ones lower tokens.
struct Shortlist {
    float v = -__builtin_inff();
    int i = INT_MAX;
    // x, of all lanes alike, takes its place.
    __device__ __forceinline__ void insert(float x, int xi)
    {
        const int lane = threadIdx.x & 63, at = __popcll(__ballot(v > x || (v == x && i < xi)));
        const float ov = __shfl_up(v, 1);
        const int oi = __shfl_up(i, 1);
        if (lane > at) {
            v = ov;
            i = oi;
        }
        if (lane == at) {
            v = x;
            i = xi;
        }
    }
};

// The n-th largest of the lanes' values, -inf if there are fewer (NaN counts as above all).
__device__ __forceinline__ float nth_largest(float x, int n)
{
    const uint32_t u = __float_as_uint(x), key = u & 0x80000000u ? ~u : u | 0x80000000u;   // ordered as the numbers
    uint32_t t = 0;
    for (int b = 31; b >= 0; --b)
        if (__popcll(__ballot(key >= (t | 1u << b))) >= n) t |= 1u << b;
    return __uint_as_float(t & 0x80000000u ? t & 0x7fffffffu : ~t);
}

// A wave goes through its part of a row in order, 64 x 16 bytes a step, kBeamAhead steps requested at a time.
//   sum         of exp(x - ref): ref is the largest logit of the first steps, and moves where one is more than 80 above it (rare).  Those of 16 bytes
//               are added in fp32 and their sums in fp64, as thousands of terms follow each other
//   shortlist   a step whose largest logit is not above the last on the list (and not below what `keep` lanes have in the first steps) costs one
//               comparison; each logit that is takes a turn of the wave.  About keep * (2 + log(steps)) turns of 80 cycles where logits come in no order
// NaN and +inf, which are no candidates, would show in the sum: then the wave goes through its part once more and takes them as -inf.
// Bound by the bytes and, at 16 bits, by the vector units (about 9 instructions a logit, 4 of them the exponential's).
constexpr int kBeamAhead = 4;

template <typename T>
__global__ __launch_bounds__(256) void k_beam_rows(BeamArgs a)
{
    typedef LogitVector<T> Vec;
    constexpr int N = Vec::N, NW = 4;
    __shared__ float s_v[NW * kBeamMax], s_ref[NW];
    __shared__ int s_i[NW * kBeamMax];
    __shared__ double s_sum[NW];
    const int row = blockIdx.y, slice = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    if (a.ended && a.ended[row]) return;
    const T* x = (const T*)a.logits + (int64_t)row * a.row_stride;
    const int mis = (int)((uintptr_t)x & 15) / (int)sizeof(T);   // elements of the first 16 bytes that are before the row
    const int64_t steps_all = ((int64_t)mis + a.vocab + 64 * N - 1) / (64 * N), workers = (int64_t)a.slices * NW, me = (int64_t)slice * NW + wave;
    const int first = (int)(steps_all * me / workers), end = (int)(steps_all * (me + 1) / workers);

    Shortlist list;
    float ref = 0.f;
    double sum = 0;
    // step s: 16 bytes a lane; at the row's ends element by element, -inf beside it
    auto load = [&](int s, u32x4& r) {
        const int64_t e0 = (int64_t)s * (64 * N) - mis;
        const int64_t e = e0 + lane * N;
        if (e0 >= 0 && e0 + 64 * N <= a.vocab) {
            r = __builtin_nontemporal_load((const u32x4*)(x + e));
            return;
        }
        T part[N];
#pragma unroll
        for (int i = 0; i < N; ++i) part[i] = e + i >= 0 && e + i < a.vocab ? x[e + i] : (T)(-__builtin_inff());
        r = __builtin_bit_cast(u32x4, part);
    };
    auto pass = [&](auto clean_pass) {
        constexpr bool CLEAN = decltype(clean_pass)::value;
        list = Shortlist{};
        sum = 0;
        auto open = [&](const u32x4& r, float (&v)[N]) {
            Vec::open(r, v);
            if constexpr (CLEAN)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (!(v[i] <= 3.4028235e38f)) v[i] = -__builtin_inff();
        };
        auto largest = [&](const float (&v)[N]) {
            float m = v[0];
#pragma unroll
            for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
            return m;
        };
        u32x4 now[kBeamAhead], next[kBeamAhead];
#pragma unroll
        for (int k = 0; k < kBeamAhead; ++k) {
            next[k] = u32x4{0, 0, 0, 0};
            if (first + k < end) load(first + k, next[k]);
        }
        float mine = -__builtin_inff();
#pragma unroll
        for (int k = 0; k < kBeamAhead; ++k)
            if (first + k < end) {
                float v[N];
                open(next[k], v);
                mine = fmaxf(mine, largest(v));
            }
        ref = fmaxf(wave_max(mine), -3.0e38f);
        // what is below the keep-th of the lanes' largest is not among the wave's keep best; `above`: only what is above it can be
        const float floor = nth_largest(mine, a.keep);
        float above = floor > -3.4028235e38f ? -__builtin_inff() : floor, last_v = -__builtin_inff();
        int last_i = INT_MAX;
        if (floor > -3.4028235e38f) {   // the next number below
            const uint32_t u = __float_as_uint(floor);
            above = __uint_as_float(u == 0 || u == 0x80000000u ? 0x80000001u : u & 0x80000000u ? u + 1 : u - 1);
        }
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
                if (__any(top > ref + 80.f)) {
                    const float moved = wave_max(top);
                    sum *= exp2((double)(ref - moved) * (double)kLog2e);
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
                if (!__any(top > above)) continue;
                const int token = (int)((int64_t)(s + k) * (64 * N) - mis) + lane * N;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    uint64_t turn = __ballot(v[i] > above);
                    while (turn) {
                        const int l = __ffsll((unsigned long long)turn) - 1;
                        list.insert(__int_as_float(__builtin_amdgcn_readlane(__float_as_int(v[i]), l)), __builtin_amdgcn_readlane(token + i, l));
                        last_v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(list.v), a.keep - 1));
                        last_i = __builtin_amdgcn_readlane(list.i, a.keep - 1);
                        turn &= turn - 1;
                        turn &= __ballot(v[i] > last_v || (v[i] == last_v && token + i < last_i));
                    }
                }
                above = fmaxf(above, last_v);
            }
        }
        sum = wave_sum(sum);
        return fabs(sum) <= 1e300;
    };
    if (!pass(std::false_type{})) pass(std::true_type{});

    // the waves' together
    if (lane < a.keep) {
        s_v[wave * a.keep + lane] = list.v;
        s_i[wave * a.keep + lane] = list.i;
    }
    if (lane == 0) {
        s_ref[wave] = ref;
        s_sum[wave] = sum;
    }
    __syncthreads();
    float* out = a.part + ((int64_t)row * a.slices + slice) * beam_part_floats(a.keep);
    if (t == 0) {
        float top = s_ref[0];
        for (int w = 1; w < NW; ++w) top = fmaxf(top, s_ref[w]);
        double all = 0;
        for (int w = 0; w < NW; ++w) all += s_sum[w] * exp2((double)(s_ref[w] - top) * (double)kLog2e);
        out[0] = top;
        *(double*)(out + 2) = all;
    }
    const int n = NW * a.keep;
    if (t >= n) return;
    const float v = s_v[t];
    const int i = s_i[t];
    int before = 0;   // entries without a candidate, all alike, keep their order
    for (int k = 0; k < n; ++k) before += s_v[k] > v || (s_v[k] == v && (s_i[k] < i || (s_i[k] == i && k < t)));
    if (before < a.keep) {
        out[4 + before] = v;
        out[4 + a.keep + before] = __int_as_float(i == INT_MAX ? -1 : i);
    }
}

// Tokens of a beam of this length, and with one more.
__device__ __forceinline__ int beam_length(int length, bool more) { return min(max(length, 0), INT_MAX - more) + more; }

// Up to kBeamRanked candidates find their places by counting those before them; more (then a row is one slice) are taken one by one, a lane of
// the first wave holding the best of its beam that is left.
__global__ __launch_bounds__(256) void k_beam_pick(BeamArgs a)
{
    __shared__ double s_top[kBeamMax], s_log[kBeamMax], s_total[kBeamMax], s_power[kBeamMax], s_rank[kBeamRanked];
    __shared__ uint64_t s_key[kBeamRanked];   // beam and token: of equal ranks the lower one is first
    __shared__ int s_over[kBeamMax], s_row[kBeamMax], s_token[kBeamMax];
    const int g = blockIdx.x, t = threadIdx.x, per = beam_part_floats(a.keep), lists = a.slices * a.keep, n = a.beams * lists;
    constexpr uint64_t kNone = ~0ull;
    if (t < a.beams) {
        const int row = g * a.beams + t;
        const bool over = a.ended && a.ended[row];
        const float* p = a.part + (int64_t)row * a.slices * per;
        double m = -__builtin_inf(), l = 0;
        if (!over) {
            for (int c = 0; c < a.slices; ++c) m = fmax(m, (double)p[c * per]);
            for (int c = 0; c < a.slices; ++c) l += *(const double*)(p + c * per + 2) * exp((double)p[c * per] - m);
        }
        s_over[t] = over;
        s_top[t] = m;
        s_log[t] = log(l);
        s_total[t] = a.totals[row];
        s_power[t] = a.power != 0.f ? pow((double)max(beam_length(a.lengths[row], !over), 1), (double)a.power) : 1.0;
    }
    if (t < a.keep) s_row[t] = s_token[t] = -1;
    __syncthreads();
    // the e-th candidate of a beam: its rank, and its sum
    auto candidate = [&](int beam, int e, double* sum, uint64_t* key) {
        *key = kNone;
        *sum = -__builtin_inf();
        if (!(fabs(s_total[beam]) <= 3.5e38)) return -__builtin_inf();
        if (s_over[beam]) {
            if (e > 0) return -__builtin_inf();
            *sum = s_total[beam];
            *key = (uint64_t)beam << 32 | (uint32_t)max(a.end_id, 0);
        } else {
            const float* p = a.part + (((int64_t)g * a.beams + beam) * a.slices + e / a.keep) * per + 4 + e % a.keep;
            const int token = __float_as_int(p[a.keep]);
            if (token < 0) return -__builtin_inf();
            *sum = s_total[beam] + (((double)p[0] - s_top[beam]) - s_log[beam]);
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
        if (a.next_lengths) a.next_lengths[at] = beam_length(a.lengths[row], !over);
        if (a.next_ended) a.next_ended[at] = over || token == a.end_id;
    };
    if (n <= kBeamRanked) {
        double sums[kBeamRanked / 256];
        for (int c = t, k = 0; c < n; c += 256, ++k) s_rank[c] = candidate(c / lists, c % lists, &sums[k], &s_key[c]);
        __syncthreads();
        for (int c = t, k = 0; c < n; c += 256, ++k) {
            const double r = s_rank[c];
            const uint64_t key = s_key[c];
            if (key == kNone) continue;
            int before = 0;
            for (int o = 0; o < n; ++o) before += s_key[o] != kNone && (s_rank[o] > r || (s_rank[o] == r && s_key[o] < key));
            if (before < a.keep) take(before, key, sums[k]);
        }
    } else if (t < 64) {
        int at = 0;
        double sum = 0, rank = -__builtin_inf();
        uint64_t key = kNone;
        if (t < a.beams) rank = candidate(t, 0, &sum, &key);
        for (int place = 0; place < a.keep; ++place) {
            double r = key == kNone ? -__builtin_inf() : rank;
            uint64_t best = key;
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) {
                const double o = __shfl_xor(r, d);
                const uint64_t ok = __shfl_xor((unsigned long long)best, d);
                if (ok != kNone && (best == kNone || o > r || (o == r && ok < best))) {
                    r = o;
                    best = ok;
                }
            }
            if (best == kNone) break;
            if (key == best) {
                take(place, key, sum);
                rank = ++at < lists ? candidate(t, at, &sum, &key) : (key = kNone, 0.0);
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
    const int width = a.next_history_stride;
    for (int k = 0; k < a.keep; ++k) {
        const int row = s_row[k], len = row < 0 ? 0 : max(a.lengths[row], 0), token = s_token[k], kept = min(len, a.history_stride);
        const int32_t* from = a.history + (int64_t)max(row, 0) * a.history_stride;
        int32_t* to = a.next_history + ((int64_t)g * a.keep + k) * width;
#pragma unroll 4
        for (int i = t; i < width; i += 256) to[i] = i < kept ? from[i] : i == len ? token : -1;
    }
}

void launch_beam_select(const BeamArgs& a, int dtype, hipStream_t s)
{
    const dim3 grid(a.slices, a.n_groups * a.beams);
    if (dtype == kF32) k_beam_rows<float><<<grid, 256, 0, s>>>(a);
    else if (dtype == kF16) k_beam_rows<_Float16><<<grid, 256, 0, s>>>(a);
    else k_beam_rows<__bf16><<<grid, 256, 0, s>>>(a);
    k_beam_pick<<<a.n_groups, 256, 0, s>>>(a);
}

}  // namespace ss

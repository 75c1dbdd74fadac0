// Kernels of beam search: of all continuations of a group's beams the best ones.
#include <climits>
#include <type_traits>

#include "ss_device.h"
#include "ss_plan.h"

namespace ss {

// Two launches.  Chunks of kBeamChunk logits of a row: their largest, the sum of the others' exponentials relative to it, and the `keep` largest with their
// tokens (no candidate behind those of its own beam can be taken, and no row has more than `keep` taken).  Then a workgroup per group: the rows' log
// sums in float64 from the chunks', candidates' ranks in float64, and their order.
__device__ __forceinline__ float logit(const float* p) { return *p; }
__device__ __forceinline__ float logit(const _Float16* p) { return (float)*p; }
__device__ __forceinline__ float logit(const __bf16* p) { return (float)*p; }

// Of two candidates the better one: larger, of equal ones the lower index (INT_MAX: none).
template <typename V>
struct Best {
    V v;
    int64_t i;
    __device__ __forceinline__ void take(V ov, int64_t oi)
    {
        if (ov > v || (ov == v && oi < i)) {
            v = ov;
            i = oi;
        }
    }
};

template <typename V>
__device__ __forceinline__ Best<V> block_best(Best<V> b, Best<V>* lds)   // 256 threads; lds: 4
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const V ov = __shfl_xor(b.v, d);
        const int64_t oi = __shfl_xor(b.i, d);
        b.take(ov, oi);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = b;
    __syncthreads();
    for (int w = 0; w < 4; ++w) b.take(lds[w].v, lds[w].i);
    return b;
}

// Tokens of a beam of this length, and with one more.
__device__ __forceinline__ int beam_length(int length, bool more) { return min(max(length, 0), INT_MAX - more) + more; }

template <typename T>
__global__ __launch_bounds__(256) void k_beam_rows(BeamArgs a)
{
    constexpr int E = kBeamChunk / 256;
    __shared__ Best<float> s_best[4];
    __shared__ float s_red[4];
    const int row = blockIdx.y, chunk = blockIdx.x, t = threadIdx.x;
    if (a.ended && a.ended[row]) return;
    const T* x = (const T*)a.logits + (int64_t)row * a.row_stride;
    const int first = chunk * kBeamChunk;
    float v[E], top = -__builtin_inff();
#pragma unroll
    for (int k = 0; k < E; ++k) {
        const int i = first + 256 * k + t;
        v[k] = i < a.vocab ? logit(x + i) : -__builtin_inff();
        if (!(fabsf(v[k]) <= 3.4028235e38f)) v[k] = -__builtin_inff();   // no candidate
        top = fmaxf(top, v[k]);
    }
    top = wave_max(top);
    if ((t & 63) == 0) s_red[t >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
    __syncthreads();
    float sum = 0.f;
    if (top > -__builtin_inff())
#pragma unroll
        for (int k = 0; k < E; ++k) sum += __builtin_amdgcn_exp2f((v[k] - top) * 1.44269504088896341f);
    sum = wave_sum(sum);
    if ((t & 63) == 0) s_red[t >> 6] = sum;
    __syncthreads();
    float* out = a.part + ((int64_t)row * a.chunks + chunk) * (2 + 2 * a.keep);
    if (t == 0) {
        out[0] = top;
        out[1] = (s_red[0] + s_red[1]) + (s_red[2] + s_red[3]);
    }
    for (int n = 0; n < a.keep; ++n) {
        Best<float> b{-__builtin_inff(), INT_MAX};
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (v[k] > -__builtin_inff()) b.take(v[k], first + 256 * k + t);
        b = block_best(b, s_best);
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (first + 256 * k + t == b.i) v[k] = -__builtin_inff();
        if (t == 0) {
            out[2 + n] = b.v;
            out[2 + a.keep + n] = __int_as_float(b.i == INT_MAX ? -1 : (int)b.i);
        }
    }
}

__global__ __launch_bounds__(256) void k_beam_pick(BeamArgs a)
{
    __shared__ Best<double> s_best[4];
    __shared__ double s_top[kBeamMax], s_log[kBeamMax], s_total[kBeamMax], s_power[kBeamMax];
    __shared__ int s_row[kBeamMax], s_token[kBeamMax];
    const int g = blockIdx.x, t = threadIdx.x, per = 2 + 2 * a.keep;
    if (t < a.beams) {
        const int row = g * a.beams + t;
        const bool ended = a.ended && a.ended[row];
        const float* p = a.part + (int64_t)row * a.chunks * per;
        double m = -__builtin_inf(), l = 0;
        if (!ended) {
            for (int c = 0; c < a.chunks; ++c) m = fmax(m, (double)p[(int64_t)c * per]);
            for (int c = 0; c < a.chunks; ++c)
                if (p[(int64_t)c * per + 1] > 0.f) l += (double)p[(int64_t)c * per + 1] * exp((double)p[(int64_t)c * per] - m);
        }
        s_top[t] = m;
        s_log[t] = log(l);
        s_total[t] = a.totals[row];
        s_power[t] = a.power != 0.f ? pow((double)max(beam_length(a.lengths[row], !ended), 1), (double)a.power) : 1.0;
    }
    __syncthreads();
    const int n = a.beams * a.chunks * a.keep;
    double last_v = __builtin_inf();
    int64_t last_i = -1;
    for (int k = 0; k < a.keep; ++k) {   // the best behind the last one taken
        Best<double> b{-__builtin_inf(), INT64_MAX};
        double sum = 0;
        for (int e = t; e < n; e += 256) {
            const int beam = e / (a.chunks * a.keep), rest = e % (a.chunks * a.keep), row = g * a.beams + beam;
            if (!(fabs(s_total[beam]) <= 3.5e38)) continue;
            double v;
            int64_t i;
            if (a.ended && a.ended[row]) {
                if (rest > 0) continue;
                v = s_total[beam] / s_power[beam];
                i = (int64_t)beam * a.vocab + max(a.end_id, 0);
            } else {
                const float* p = a.part + ((int64_t)row * a.chunks + rest / a.keep) * per + 2 + rest % a.keep;
                const int token = __float_as_int(p[a.keep]);
                if (token < 0) continue;
                v = (s_total[beam] + (((double)p[0] - s_top[beam]) - s_log[beam])) / s_power[beam];
                i = (int64_t)beam * a.vocab + token;
            }
            if (v < last_v || (v == last_v && i > last_i)) b.take(v, i);
        }
        b = block_best(b, s_best);
        last_v = b.v;
        last_i = b.i;
        if (t == 0) {
            const int at = g * a.keep + k, none = b.i == INT64_MAX, beam = none ? 0 : (int)(b.i / a.vocab), row = g * a.beams + beam;
            const bool over = !none && a.ended && a.ended[row];
            const int token = none ? -1 : over ? a.end_id : (int)(b.i % a.vocab);
            sum = none ? -__builtin_inf() : b.v;
            if (!none) {   // the sum again, without the length
                sum = s_total[beam];
                if (!over) {
                    const float* p = a.part + ((int64_t)row * a.chunks + token / kBeamChunk) * per + 2;
                    for (int c = 0; c < a.keep; ++c)
                        if (__float_as_int(p[a.keep + c]) == token) sum = s_total[beam] + (((double)p[c] - s_top[beam]) - s_log[beam]);
                }
            }
            s_row[k] = none ? -1 : row;
            s_token[k] = over ? -1 : token;   // to be appended
            a.parent[at] = none ? -1 : row;
            a.token[at] = token;
            a.next_totals[at] = (float)sum;
            if (a.next_lengths) a.next_lengths[at] = none ? 0 : beam_length(a.lengths[row], !over);
            if (a.next_ended) a.next_ended[at] = none || over || token == a.end_id;
        }
    }
    if (!a.next_history) return;
    __syncthreads();
    for (int k = 0; k < a.keep; ++k) {
        const int row = s_row[k], len = row < 0 ? 0 : max(a.lengths[row], 0), token = s_token[k];
        for (int i = t; i < a.next_history_stride; i += 256) {
            int x = -1;
            if (i < len && i < a.history_stride) x = a.history[(int64_t)row * a.history_stride + i];
            else if (i == len) x = token;
            a.next_history[((int64_t)g * a.keep + k) * a.next_history_stride + i] = x;
        }
    }
}

void launch_beam_select(const BeamArgs& a, int dtype, hipStream_t s)
{
    const dim3 grid(a.chunks, a.n_groups * a.beams);
    if (dtype == kF32) k_beam_rows<float><<<grid, 256, 0, s>>>(a);
    else if (dtype == kF16) k_beam_rows<_Float16><<<grid, 256, 0, s>>>(a);
    else k_beam_rows<__bf16><<<grid, 256, 0, s>>>(a);
    k_beam_pick<<<a.n_groups, 256, 0, s>>>(a);
}

}  // namespace ss

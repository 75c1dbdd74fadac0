// Device helpers that the kernels share: conversions, the packed layout, sums and maxima over lanes.
#ifndef SS_DEVICE_H
#define SS_DEVICE_H

#include <hip/hip_runtime.h>

#include "ss_kernels.h"

namespace ss {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));  // one 16-byte operand fragment

// ------------------------------------------------------------------------------------------ helpers
__device__ __forceinline__ float bf2f(bf16_t b) { return __uint_as_float(((uint32_t)b) << 16); }

__device__ __forceinline__ bf16_t f2bf(float f)
{
    uint32_t u = __float_as_uint(f);
    u += 0x7FFFu + ((u >> 16) & 1u);  // round to nearest, ties to even (inputs are finite)
    return (bf16_t)(u >> 16);
}

// Both operands of every projection are IEEE half.  A bf16 weight keeps its exact value in that format (8
// significand bits fit in 11; see k_pack_weight for the two ends of the range).  An activation that feeds a
// projection is rounded to half once: 11 significand bits, where a bf16 operand would keep 8 - one such rounding
// per projection input, six per layer over 32+ layers, is the dominant term of the logit error, and at 8 bits it
// is as large as the whole tolerance.  Finite values saturate, like the key/value slots below; a NaN stays a NaN.
__device__ __forceinline__ f16_t f2h(float f)
{
    const float c = fminf(fmaxf(f, -65504.f), 65504.f);   // of a NaN and a number these return the number
    return __builtin_bit_cast(f16_t, (_Float16)(f != f ? f : c));
}

// Rotation of a pair of elements.  Which product of the sum is rounded first is written out: the compiler would choose by what is around
// it, and every kernel that rotates is to round alike (a prompt's keys and queries do not depend on whether q|k|v was cut in k-slices).
// In the difference it rounds the second product in all of them.
__device__ __forceinline__ float2 rotated(float a, float b, float cs, float sn)
{
    return make_float2(a * cs - b * sn, fmaf(b, cs, a * sn));
}

// Key/value slots are stored as IEEE half: the same 2 bytes per element as bf16 with three more
// significand bits; keys and values are projections of RMS-normalised activations, far inside its range.
__device__ __forceinline__ float kv2f(kv_t b) { return (float)__builtin_bit_cast(_Float16, b); }
// Saturating: a value beyond the half range is stored as the largest finite half, never as infinity (an infinite
// key would turn the softmax into NaN and the token choice into an arbitrary id).
__device__ __forceinline__ kv_t f2kv(float f)
{
    return __builtin_bit_cast(kv_t, (_Float16)fminf(fmaxf(f, -65504.f), 65504.f));
}

// Element (r, k) of a packed [rows, Kp] matrix.
__device__ __forceinline__ size_t pk_index(int r, int k, int Kp)
{
    return ((size_t)(r >> 4) * (size_t)(Kp >> 5) + (size_t)(k >> 5)) * 512u +
           (size_t)(((((k & 31) >> 3) << 4) + (r & 15)) * 8 + (k & 7));
}

// Output strips of q, k and v are packed in pairs: a head's strip i of its first half (elements 16i..16i+15) and its
// strip i of the second half are neighbours, so that the two elements of a rotation pair (e, e + hd/2) are in the same
// lane of whichever wave computes them, as gate and up are.  qkv_strip: natural strip -> packed strip; qkv_col: column of
// element e < hd/2 of a head in the projection's output (its partner follows 16 columns later).
__device__ __forceinline__ int qkv_strip(int strip, int head_strips)
{
    const int h = strip / head_strips, i = strip - h * head_strips, half = head_strips >> 1;
    return h * head_strips + (i < half ? 2 * i : 2 * (i - half) + 1);
}
__device__ __forceinline__ int qkv_col(int e) { return (e >> 4) * 32 + (e & 15); }

// v of another lane of the same row of 16 lanes (a DPP control), at the cost of a register move.
template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;
constexpr int kDppRotate4 = 0x124, kDppRotate8 = 0x128;

// op(v, v of the lane M = 16 or 32 away), M being a bit of the lane's number: two rows or halves of the wave change places,
// which takes no trip through LDS as a general shuffle does (the norms and the decode attention are chains of such latencies:
// with general shuffles, decode of 7B, one row, 24 steps 64.3 ms instead of 63.5, 16 rows 79.6 / 78.9, 51 rows 58.4 / 57.8).
template <int M, typename Op>
__device__ __forceinline__ float across(float v, Op op)
{
    const unsigned u = (unsigned)__float_as_int(v);
    const auto r = M == 32 ? __builtin_amdgcn_permlane32_swap(u, u, false, false) : __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return op(__int_as_float((int)r[0]), __int_as_float((int)r[1]));
}
struct Add { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct Max { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

// Over the wave, in each lane: lanes 32, 16, 8, 4, 2 and 1 apart in turn (after a step the lanes that it joined are alike, so
// that a turn by 4 in a row of 16 does for 4 apart).
template <typename Op>
__device__ __forceinline__ float wave_all(float v, Op op)
{
    v = across<16>(across<32>(v, op), op);
    v = op(v, dpp<kDppRotate8>(v));
    v = op(v, dpp<kDppRotate4>(v));
    v = op(v, dpp<kDppXor2>(v));
    return op(v, dpp<kDppXor1>(v));
}
__device__ __forceinline__ float wave_sum(float v) { return wave_all(v, Add()); }
__device__ __forceinline__ float wave_max(float v) { return wave_all(v, Max()); }

// Sum over a group of 8 or 16 neighbouring lanes, in each of them.
template <int N>
__device__ __forceinline__ float group_sum(float v)
{
    static_assert(N == 8 || N == 16, "half a row or a row");
    v += dpp<kDppXor1>(v);
    v += dpp<kDppXor2>(v);
    v += dpp<kDppHalfMirror>(v);   // the lanes of four are alike by now
    if (N == 16) v += dpp<kDppMirror>(v);
    return v;
}

// Place of a slot of a tile of 64 in its staged V^T rows: a lane's 8 slots of two 16-slot score tiles are neighbours.
__device__ __forceinline__ int vt_pos(int k) { return (k & 32) + ((k >> 2) & 3) * 8 + ((k >> 4) & 1) * 4 + (k & 3); }

// 16 bytes per lane straight into LDS: the wave's 64 pieces land behind each other at slot + place, from base + lane_off.
// The copies are written in assembly because the compiler would wait for all of them before every LDS read: it counts
// only its own loads, and the waits here are written out.  They name no output register; waits that the compiler adds
// for loads of its own can only be too strict.
__device__ __forceinline__ void lds_copy_1k(unsigned slot, unsigned place, const void* base, unsigned lane_off)
{
    asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3" ::"s"(slot), "s"(place), "v"(lane_off), "s"(base)
                 : "memory", "scc");
}

// At most N copies of this wave are still on their way, its LDS reads are done, and then so are every other wave's.  The
// builtin tells the compiler that the operands read before are in their registers (after a wait in assembly it would wait
// for each of them once more).
template <int N>
__device__ __forceinline__ void wait_copies_and_meet()
{
    static_assert(N < 64, "the counter has 6 bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));   // vmcnt(N) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
}

}  // namespace ss

#endif

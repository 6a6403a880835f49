// Sums and maxima over neighbouring lanes of a wavefront, every lane of the group getting the result. Not installed.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ficco {

// Inside 16 lanes the values travel as operands of the vector instructions themselves (DPP: mirrored rows, mirrored halves, swaps
// inside four lanes), between rows of 16 and halves of 32 by v_permlane16/32_swap. (The LDS crossbar behind __shfl_xor takes about
// a hundred cycles a step.) Every step adds the same two numbers in both lanes, so all lanes get the same bits.
template <int CTRL>
static __device__ __forceinline__ float dpp(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
template <int LANES, class Op>
static __device__ __forceinline__ float over_lanes(float v, Op op)
{
    static_assert(LANES == 8 || LANES == 16 || LANES == 32 || LANES == 64, "lanes of a group");
    if constexpr (LANES >= 16) v = op(v, dpp<0x140>(v));       // row_mirror
    v = op(v, dpp<0x141>(v));                                   // row_half_mirror
    v = op(v, dpp<0x4E>(v));                                    // quad_perm [2,3,0,1]
    v = op(v, dpp<0xB1>(v));                                    // quad_perm [1,0,3,2]
    if constexpr (LANES >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if constexpr (LANES >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return v;
}
template <int LANES>
static __device__ __forceinline__ float lane_sum(float v) { return over_lanes<LANES>(v, [](float a, float b) { return a + b; }); }
template <int LANES>
static __device__ __forceinline__ float lane_max(float v) { return over_lanes<LANES>(v, [](float a, float b) { return fmaxf(a, b); }); }

// Sums of N values over TPR threads (whole wavefronts, all of the workgroup if more than one), every thread getting them. `s`:
// N * 16 floats that no wavefront may still read from an earlier call.
template <int TPR, int N>
static __device__ __forceinline__ void thread_sums(float (&v)[N], float *s)
{
    constexpr int W = TPR / 64;
    static_assert(TPR % 64 == 0 && W <= 16, "whole wavefronts");
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lane_sum<64>(v[k]);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) s[k * 16 + (threadIdx.x >> 6)] = v[k];
        __syncthreads();
        const int w = threadIdx.x & 15;
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = lane_sum<16>(w < W ? s[k * 16 + w] : 0.f);
    }
}

// Sum over k in [0, n) of in[k * stride] by a workgroup of 1024 threads: 32 columns side by side (`in` is the thread's, column threadIdx.x
// % 32; there: it exists), 32 slices of k, joined through LDS (`s`: 32 x 32 floats) in the order of the slices. The first 32
// threads have the sums.
static __device__ __forceinline__ float column_sum(const float *in, int n, int64_t stride, bool there, float (*s)[32])
{
    const int col = threadIdx.x & 31, slice = threadIdx.x >> 5;
    float t = 0.f;
    if (there)
#pragma unroll 8
        for (int k = slice; k < n; k += 32) t += in[(int64_t)k * stride];
    s[slice][col] = t;
    __syncthreads();
    if (slice) return 0.f;
#pragma unroll
    for (int k = 1; k < 32; ++k) t += s[k][col];
    return t;
}

}  // namespace ficco

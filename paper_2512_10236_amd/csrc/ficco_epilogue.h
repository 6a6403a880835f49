// What the linear operator does between its product and its result, and the slopes its backward pass needs. Not installed.
#pragma once
#include "../../include/ficco.h"
#include "ficco_tile.h"

namespace ficco {

// z = acc + bias, pre = bf16(z), C = act(z) + residual; any of bias, pre and residual may be null. Strides in elements.
struct Epilogue {
    const void *bias;             // [N], bf16 or fp32
    const uint16_t *residual;
    uint16_t *pre;
    int64_t ld_residual, ld_pre;
    int32_t activation, bias_f32;
};

static __device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
static __device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }

// 1 / (1 + 2^-x): v_exp_f32 and v_rcp_f32, one unit in the last place each, no division
static __device__ __forceinline__ float sigmoid2(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-x)); }

constexpr float kLog2E = 1.44269504f, kGeluC = 0.7978845608f /* sqrt(2/pi) */, kGeluCube = 0.044715f;

// Phi(-|z|), the normal distribution function's lower tail: erfc(x) exp(x^2), x = |z|/sqrt(2), is smooth in t = 1/(1 + 0.44 x),
// which maps [0, inf) to (0, 1]; the polynomial is a weighted least-squares fit of its own over x in [0, 10], off by 2e-7
// of the value; in fp32 that is 5e-7 down to z = -1 and, by the exponent's rounding, 2e-6 at -6, where the value is 1e-9, and 3e-6 at -8.
static __device__ __forceinline__ float normal_tail(float z)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.44f * 0.70710678f, 1.0f));
    float q = 0.07122400f;
    q = fmaf(q, t, -0.27795024f);
    q = fmaf(q, t, 0.29669131f);
    q = fmaf(q, t, -0.020184173f);
    q = fmaf(q, t, 0.21581407f);
    q = fmaf(q, t, 0.21731301f);
    q = fmaf(q, t, 0.24887127f);
    q = fmaf(q, t, 0.24822095f);
    return 0.5f * (q * t) * __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2E));
}

template <int ACT>
static __device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == FICCO_ACT_RELU) return z > 0.f ? z : z != z ? z : 0.f;
    else if constexpr (ACT == FICCO_ACT_GELU) {
        const float h = normal_tail(z);
        return z * (z < 0.f ? h : 1.0f - h);
    } else if constexpr (ACT == FICCO_ACT_GELU_TANH) {       // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
        return z * sigmoid2(z * fmaf(z * z, 2.0f * kLog2E * kGeluC * kGeluCube, 2.0f * kLog2E * kGeluC));
    } else if constexpr (ACT == FICCO_ACT_SILU) return z * sigmoid2(z * kLog2E);
    else return z;
}

// act'(z). The smooth ones' slopes are 0 and 1 to the last bit beyond |z| = 32 (GELU, either) or 128 (SiLU, z exp(z) far below zero, which leaves
// fp32's normal numbers at -91); without the bound z^3 and its exponential, or z itself at infinity, would make infinity times zero of it. (NaN passes
// the comparisons.)
template <int ACT>
static __device__ __forceinline__ float slope(float z)
{
    if constexpr (ACT == FICCO_ACT_NONE) return 1.0f;
    else if constexpr (ACT == FICCO_ACT_RELU) return z > 0.f ? 1.0f : z != z ? z : 0.f;
    else {
        constexpr float far = ACT == FICCO_ACT_SILU ? 128.f : 32.f;
        z = z > far ? far : z < -far ? -far : z;
        if constexpr (ACT == FICCO_ACT_GELU) {
            const float h = normal_tail(z);
            return fmaf(z * 0.39894228f, __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2E)), z < 0.f ? h : 1.0f - h);
        } else if constexpr (ACT == FICCO_ACT_GELU_TANH) {
            const float s = sigmoid2(z * fmaf(z * z, 2.0f * kLog2E * kGeluC * kGeluCube, 2.0f * kLog2E * kGeluC));
            return fmaf(z * s * (1.0f - s), fmaf(z * z, 6.0f * kGeluC * kGeluCube, 2.0f * kGeluC), s);
        } else {
            const float s = sigmoid2(z * kLog2E);
            return s * fmaf(z, 1.0f - s, 1.0f);
        }
    }
}

// 4 values of the bias from column n on (a multiple of 4)
static __device__ __forceinline__ f32x4_t bias4(const Epilogue &e, int n)
{
    if (!e.bias) return f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (e.bias_f32) {
        const float *b = static_cast<const float *>(e.bias) + n;
        return f32x4_t{b[0], b[1], b[2], b[3]};
    }
    const uint16_t *b = static_cast<const uint16_t *>(e.bias) + n;
    return f32x4_t{__uint_as_float((uint32_t)b[0] << 16), __uint_as_float((uint32_t)b[1] << 16), __uint_as_float((uint32_t)b[2] << 16),
                   __uint_as_float((uint32_t)b[3] << 16)};
}

// Calls f(integral_constant<int, activation>): the activation is known to the compiler inside.
template <class Fn>
static __device__ __forceinline__ void with_activation(int activation, Fn &&f)
{
    switch (activation) {
    case FICCO_ACT_RELU: f(std::integral_constant<int, FICCO_ACT_RELU>{}); break;
    case FICCO_ACT_GELU: f(std::integral_constant<int, FICCO_ACT_GELU>{}); break;
    case FICCO_ACT_GELU_TANH: f(std::integral_constant<int, FICCO_ACT_GELU_TANH>{}); break;
    case FICCO_ACT_SILU: f(std::integral_constant<int, FICCO_ACT_SILU>{}); break;
    default: f(std::integral_constant<int, FICCO_ACT_NONE>{}); break;
    }
}

// 4 consecutive columns of one row, column n on: what a kernel with one row a lane does (see tile_store_epilogue for 8).
template <int ACT>
static __device__ __forceinline__ void store4(const Epilogue &e, f32x4_t z, f32x4_t bias, uint16_t *c, int64_t row, int n)
{
    typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int v = 0; v < 4; ++v) z[v] += bias[v];
    if (e.pre) *reinterpret_cast<u32x2_t *>(e.pre + row * e.ld_pre + n) = u32x2_t{pack2_bf16_rne(z[0], z[1]), pack2_bf16_rne(z[2], z[3])};
#pragma unroll
    for (int v = 0; v < 4; ++v) z[v] = activate<ACT>(z[v]);
    if (e.residual) {
        const u32x2_t r = *reinterpret_cast<const u32x2_t *>(e.residual + row * e.ld_residual + n);
        z[0] += bf16_lo(r[0]); z[1] += bf16_hi(r[0]); z[2] += bf16_lo(r[1]); z[3] += bf16_hi(r[1]);
    }
    *reinterpret_cast<u32x2_t *>(c) = u32x2_t{pack2_bf16_rne(z[0], z[1]), pack2_bf16_rne(z[2], z[3])};
}

// tile_store with an epilogue: the exchange between lanes is made with the fp32 values, so that a lane has 8 consecutive
// columns of a row before bias, activation and residual are applied and everything it reads and writes there is 16 bytes.
// row0, col0: the tile's place. M 16384, K 8192, N 3584: nothing 709 us, SiLU 717, GELU by tanh 722, by erf 746.
template <class T, int ACT>
static __device__ __forceinline__ void tile_store_epilogue(const TileAcc<T> &ta, const Epilogue &e, uint16_t *c_tile, int rows_valid,
                                                           int cols_valid, int64_t ldc, int64_t row0, int col0)
{
    const f32x4_t (&acc)[T::FN][T::FM] = ta.acc;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / T::WGN, wn = wave % T::WGN;
    const int frow = lane & 15, fh = lane >> 4;
    const int n0 = wn * T::WTN + (fh & 1) * 16 + (fh >> 1) * 8;
    f32x4_t bias[T::FN];
#pragma unroll
    for (int j = 0; j < T::FN; j += 2) {
        const int n = n0 + j * 16;
        const bool there = n < cols_valid;
        bias[j] = there ? bias4(e, col0 + n) : f32x4_t{0.f, 0.f, 0.f, 0.f};
        bias[j + 1] = there ? bias4(e, col0 + n + 4) : f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    // All of the residual's values before the first store (the fragments' registers are free by now): vector memory operations
    // complete in order, so a load behind a store waits for that store.
    u32x4_t res[T::FM][T::FN / 2];
    if (e.residual) {
        const uint16_t *r0 = e.residual + row0 * e.ld_residual + col0;
#pragma unroll
        for (int i = 0; i < T::FM; ++i) {
            const uint16_t *r = r0 + (int64_t)min(wm * T::WTM + i * 16 + frow, rows_valid - 1) * e.ld_residual;
#pragma unroll
            for (int j = 0; j < T::FN; j += 2) res[i][j / 2] = *reinterpret_cast<const u32x4_t *>(r + min(n0 + j * 16, cols_valid - 8));
        }
    }
    static_for<T::FM>([&](auto i_c) __attribute__((always_inline)) {
        constexpr int i = decltype(i_c)::value;
        const int m = wm * T::WTM + i * 16 + frow;
        uint16_t *crow = c_tile + (int64_t)m * ldc;
        static_for<T::FN / 2>([&](auto j_c) __attribute__((always_inline)) {
            constexpr int j = 2 * decltype(j_c)::value;
            float z[8];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[j][i][v]), __float_as_uint(acc[j + 1][i][v]), false, false);
                z[v] = __uint_as_float(x[0]) + bias[j][v];
                z[4 + v] = __uint_as_float(x[1]) + bias[j + 1][v];
            }
            const int n = n0 + j * 16;
            if (m < rows_valid && n < cols_valid) {
                if (e.pre)
                    *reinterpret_cast<u32x4_t *>(e.pre + (row0 + m) * e.ld_pre + col0 + n) =
                        u32x4_t{pack2_bf16_rne(z[0], z[1]), pack2_bf16_rne(z[2], z[3]), pack2_bf16_rne(z[4], z[5]), pack2_bf16_rne(z[6], z[7])};
#pragma unroll
                for (int v = 0; v < 8; ++v) z[v] = activate<ACT>(z[v]);
                if (e.residual) {
                    const u32x4_t r = res[i][j / 2];
#pragma unroll
                    for (int v = 0; v < 4; ++v) { z[2 * v] += bf16_lo(r[v]); z[2 * v + 1] += bf16_hi(r[v]); }
                }
                *reinterpret_cast<u32x4_t *>(crow + n) =
                    u32x4_t{pack2_bf16_rne(z[0], z[1]), pack2_bf16_rne(z[2], z[3]), pack2_bf16_rne(z[4], z[5]), pack2_bf16_rne(z[6], z[7])};
            }
        });
    });
}

}  // namespace ficco

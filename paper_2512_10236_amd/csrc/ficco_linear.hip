// A product with bias, activation and residual in its epilogue, and its gradients (ficco_linear, ficco_linear_backward):
//   z = A W + b,  C = act(z) + R          dZ = dC act'(z),  db = sum_m dZ,  dA = dZ W^T,  dW = A^T dZ
// The products run on the tile routine of the GEMM kernels (ficco_tile.h): bf16 in, fp32 accumulators, k ascending. The epilogue takes
// the accumulators before they are rounded, so that bias, activation and residual cost no pass over memory of their own.
//
// The backward pass is bound by its two products. What they need beside their inputs is made once by turn_kernel, a streaming
// kernel: dZ (with its column sums), and, where the products cannot read them as they are, the operands with the other index
// contiguous.
#include "ficco_linear.h"
#include "ficco_lanes.h"

namespace ficco {
namespace {

int launch_tiles(int tile, const LinearLaunch &a, hipStream_t s)
{
    switch (tile) {
#define X(id, T) case id: return launch_tiles_t<T, false, false>(a, s);
    FICCO_FOR_EACH_TILE(X)
#undef X
    default: return FICCO_ERR_ARG;
    }
}

// A choice that follows from the sizes (and the device's CUs), remembered for those that a thread asked for last: the tile rule takes
// 1.2 us of the host, of the 8 that a small call has.
template <class Choice, class Choose>
Choice remembered(int64_t M, int64_t K, int64_t N, bool kn, Choose &&choose)
{
    struct Known {
        int64_t M, K, N;
        int cus;
        bool kn;
        Choice choice;
    };
    static thread_local Known known[32];
    const int cus = compute_units();
    Known &k = known[((uint64_t)(M * 131 + K * 31 + N * 7 + kn) * 0x9E3779B97F4A7C15ull) >> 59];
    if (k.cus != cus || k.M != M || k.K != K || k.N != N || k.kn != kn) k = Known{M, K, N, cus, kn, choose()};
    return k.choice;
}

// The tile rule's answer for one launch over an M x K x N product with its operands in place, and its estimate.
struct Tile {
    int id;
    double us;
};
Tile tile_for(int64_t M, int64_t K, int64_t N)
{
    return remembered<Tile>(M, K, N, false, [&] {
        ficco_plan_t shape;
        shape.M = M; shape.K = K; shape.N = N; shape.G = 1; shape.c = 1;
        shape.schedule = FICCO_SERIAL;
        shape.order = FICCO_ORDER_STEP_MAJOR;
        shape.mode = FICCO_MODE_GEMM_ONLY;
        Tile t{0, 0};
        if (!build_lists(&shape)) t.id = choose_tile(&shape, compute_units(), false, &t.us);
        return t;
    });
}

// ------------------------------------------------------------------------------------------------------------ few rows
// A product of a few rows is the weight's way through the chip, once, and where that is short, the latency of a load and of a
// join. A workgroup has a tile of 8 AB rows x 16 NB columns and all of k, its 8 wavefronts every 8th k-tile each (128 bytes of a
// row, so that together they read 1 KiB of each row at a time). A wavefront streams its k-tiles through a ring of D stages of its
// own in LDS, without barriers: a stage is filled by loads of 8 rows x 128 bytes straight to LDS, which is what makes whole lines
// of them, and read as fragments. The eight partial tiles are added through LDS in the order of the wavefronts. So narrow tiles
// over all of k, instead of wide ones, spread the weight over as many CUs as there are.
// Fragments loaded from memory directly, a lane a row: a CU then draws 16 bytes a cycle, one lane's at a time.
template <int AB_, int NB_, bool SB_>
struct RowsCfg {
    static constexpr bool SB = SB_;                            // the weight is [K,N]
    static constexpr int AB = AB_, NB = NB_, WAVES = 8, FM = AB < 2 ? 1 : AB / 2, BM = 8 * AB, BN = 16 * NB;
    static constexpr int LOADS = AB + 2 * NB, STAGE = LOADS * 1024;              // a wavefront's, per k-tile
    static constexpr int D = 160 * 1024 / (WAVES * STAGE) < 6 ? 160 * 1024 / (WAVES * STAGE) : 6;
    static constexpr int RING = D * STAGE, PART = FM * NB * 1024;
    static constexpr int LDS_BYTES = WAVES * (RING > PART ? RING : PART);
    static_assert(D >= 2 && (D - 1) * LOADS < 64, "a ring of two stages or more, vmcnt has 6 bits");
    static_assert(!SB || NB == 2 || NB % 4 == 0, "whole lines, or halves, of a [K,N] weight's rows");
};
constexpr int kRowsThreads = 512;

// splits > 1: the workgroups of a tile share k, each a run of k-tiles, and write fp32 sums to part [splits][M][N], which
// linear_join_kernel adds in order. For a long k over few columns, where the tiles leave most CUs idle.
// One row, K 4096, N 768: 5.3 us, of which the weight from memory is 1.3.
template <class T>
__global__ __launch_bounds__(kRowsThreads) void linear_rows_kernel(LinearLaunch a, int splits, float *part)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6), j = lane & 15, g = lane >> 4;
    // tiles in 8 runs, one per XCD, rows fastest: the row tiles that read the same columns of the weight share an L2
    const int tiles_m = (a.M + T::BM - 1) / T::BM, tiles_n = (a.N + T::BN - 1) / T::BN;
    const XcdRun run = xcd_run(blockIdx.x, gridDim.x, tiles_m * tiles_n * splits);
    const int lid = run.start + run.first, rest = lid / tiles_m, split = rest % splits;
    const int row0 = lid % tiles_m * T::BM, col0 = rest / splits * T::BN;
    const int k_tiles = scalar(a.K) / kBK, KT = scalar((int)((int64_t)(split + 1) * k_tiles / splits)), kt0 = scalar((int)((int64_t)split * k_tiles / splits)) + wave;
    const uint16_t *const A = scalar_base(a.A + (int64_t)row0 * a.lda), *const W = scalar_base(a.W + (T::SB ? (int64_t)col0 : (int64_t)col0 * a.ldw));
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem + wave * T::RING;
    // 16-byte slot c of row r of 16 lies at slot c ^ ((r >> 1) & 7); rows and columns that are not there: the last that is
    uint32_t off[T::LOADS];
#pragma unroll
    for (int l = 0; l < T::LOADS; ++l) {
        if constexpr (T::SB) {
            if (l >= T::AB) {
                off[l] = strided_lane_offset<T::BN>(l - T::AB, lane, min(T::BN, a.N - col0), a.ldw);
                continue;
            }
        }
        const int r = (l < T::AB ? l : l - T::AB) * 8 + lane / 8;
        const int row = l < T::AB ? min(r, a.M - 1 - row0) : min(r, a.N - 1 - col0);
        off[l] = ((uint32_t)row * (uint32_t)(l < T::AB ? a.lda : a.ldw) + (uint32_t)(((lane % 8) ^ ((r >> 1) & 7)) * 8)) * 2u;
    }
    auto issue = [&](int kt, uint32_t stage) __attribute__((always_inline)) {
        static_for<T::LOADS>([&](auto l_c) __attribute__((always_inline)) {
            constexpr int l = decltype(l_c)::value;
            set_lds_target<l * 1024>(ring + stage);
            asm volatile("s_nop 0" ::: "memory");
            load_to_lds_16(l < T::AB ? A + (int64_t)kt * kBK : W + (T::SB ? kt * (a.ldw * kBK) : (int64_t)kt * kBK), off[l]);
        });
        __builtin_amdgcn_sched_barrier(0);
    };
    f32x4_t acc[T::FM][T::NB];
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int n = 0; n < T::NB; ++n) acc[i][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // a lane's part of a transposing read (see tile_accumulate_from)
    const int trow = 8 * g + (j >> 2);
    uint32_t t_lane = 0, t_swz = 0;
    if constexpr (T::SB) {
        t_lane = ring + T::AB * 1024 + trow * T::BN * 2 + ((j & 3) >> 1) * 16 + (j & 1) * 8;
        t_swz = strided_swizzle<T::BN>(trow) * 16;
    }
    if (kt0 < KT) {
        // past the wavefront's last k-tile the loads go on, on that k-tile again and into stages that are not read
        const int last = kt0 + (KT - 1 - kt0) / T::WAVES * T::WAVES;
#pragma unroll
        for (int d = 0; d < T::D; ++d) issue(min(kt0 + d * T::WAVES, last), d * T::STAGE);
        uint32_t stage = 0;
#pragma clang loop unroll(disable)
        for (int kt = kt0; kt < KT; kt += T::WAVES) {
            wait_vmem<(T::D - 1) * T::LOADS>();
            __builtin_amdgcn_sched_barrier(0);
            const unsigned char *const base = smem + wave * T::RING + stage;
            bf16x8_t fa[2][T::FM], fw[2][T::NB];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int slot = ((4 * h + g) ^ ((j >> 1) & 7)) << 4;
#pragma unroll
                for (int i = 0; i < T::FM; ++i) fa[h][i] = *reinterpret_cast<const bf16x8_t *>(base + (16 * i + (T::AB == 1 ? j & 7 : j)) * 128 + (T::AB == 1 ? ((4 * h + g) ^ (((j & 7) >> 1) & 7)) << 4 : slot));
#pragma unroll
                for (int n = 0; n < T::NB; ++n) {
                    if constexpr (T::SB) fw[h][n] = strided_fragment<T::BN>(stage + t_lane + h * 32 * T::BN * 2 + ((n * 32) ^ t_swz));
                    else fw[h][n] = *reinterpret_cast<const bf16x8_t *>(base + T::AB * 1024 + (16 * n + j) * 128 + slot);
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the stage has been read: it may be filled again
            __builtin_amdgcn_sched_barrier(0);
            issue(min(kt + T::D * T::WAVES, last), stage);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < T::FM; ++i)
#pragma unroll
                    for (int n = 0; n < T::NB; ++n) acc[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[h][n], fa[h][i], acc[i][n], 0, 0, 0);
            stage = stage == (T::D - 1) * T::STAGE ? 0 : stage + T::STAGE;
        }
        wait_vmem<0>();                    // no load may arrive in LDS that is used for something else
    }
    __syncthreads();
    f32x4_t *const tile = reinterpret_cast<f32x4_t *>(smem);
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int n = 0; n < T::NB; ++n) tile[(wave * T::FM * T::NB + i * T::NB + n) * 64 + lane] = acc[i][n];
    __syncthreads();
    for (int q = wave; q < T::FM * T::NB; q += T::WAVES) {
        f32x4_t z = tile[q * 64 + lane];
#pragma unroll
        for (int w = 1; w < T::WAVES; ++w) {
            const f32x4_t t = tile[(w * T::FM * T::NB + q) * 64 + lane];
#pragma unroll
            for (int v = 0; v < 4; ++v) z[v] += t[v];
        }
        // z[v] is C[row0 + 16 i + lane % 16][col0 + 16 n + 4 (lane / 16) + v]; N is a multiple of 8
        const int64_t m = row0 + 16 * (q / T::NB) + j;
        const int n = col0 + 16 * (q % T::NB) + 4 * g;
        if (m < min(a.M, row0 + T::BM) && n < a.N) {
            if (splits > 1) {
                *reinterpret_cast<f32x4_t *>(part + ((int64_t)split * a.M + m) * a.N + n) = z;
                continue;
            }
            const f32x4_t bias = bias4(a.e, n);
            with_activation(a.e.activation, [&](auto act) __attribute__((always_inline)) { store4<act.value>(a.e, z, bias, a.C + m * a.ldc + n, m, n); });
        }
    }
}

__global__ __launch_bounds__(256) void linear_join_kernel(LinearLaunch a, int splits, const float *__restrict__ part)
{
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, plane = (int64_t)a.M * a.N;
    if (at >= plane) return;
    f32x4_t z = *reinterpret_cast<const f32x4_t *>(part + at);
#pragma unroll 4
    for (int k = 1; k < splits; ++k) {
        const f32x4_t t = *reinterpret_cast<const f32x4_t *>(part + k * plane + at);
#pragma unroll
        for (int v = 0; v < 4; ++v) z[v] += t[v];
    }
    const int64_t m = at / a.N;
    const int n = (int)(at - m * a.N);
    const f32x4_t bias = bias4(a.e, n);
    with_activation(a.e.activation, [&](auto act) __attribute__((always_inline)) { store4<act.value>(a.e, z, bias, a.C + m * a.ldc + n, m, n); });
}

template <class T>
int launch_rows_t(const LinearLaunch &a, int splits, float *part, hipStream_t s)
{
    const int64_t tiles = (((int64_t)a.M + T::BM - 1) / T::BM) * (((int64_t)a.N + T::BN - 1) / T::BN) * splits;
    if (splits < 1 || (splits > 1 && !part) || tiles > 0x7FFFFFFF / kRowsThreads) return FICCO_ERR_SHAPE;
    HIP_TRY(raise_lds_limit<&linear_rows_kernel<T>>(T::LDS_BYTES));
    hipLaunchKernelGGL(linear_rows_kernel<T>, dim3((unsigned)tiles), dim3(kRowsThreads), T::LDS_BYTES, s, a, splits, part);
    HIP_TRY(hipGetLastError());
    if (splits > 1) {
        hipLaunchKernelGGL(linear_join_kernel, dim3((unsigned)(((int64_t)a.M * a.N / 4 + 255) / 256)), dim3(256), 0, s, a, splits, part);
        HIP_TRY(hipGetLastError());
    }
    return FICCO_OK;
}

// Tiles of the few-rows kernel: 8 ab rows x 16 nb columns, of an [N,K] weight or of a [K,N] one
#define FICCO_FOR_EACH_ROWS(X) \
    X(1, 1, false) X(1, 2, false) X(1, 4, false) X(2, 1, false) X(2, 2, false) X(2, 4, false) X(4, 1, false) X(4, 2, false) X(8, 1, false) \
    X(1, 2, true) X(2, 2, true) X(1, 4, true) X(2, 4, true)
int launch_rows(int ab, int nb, bool kn, const LinearLaunch &a, int splits, float *part, hipStream_t s)
{
#define X(AB, NB, SB) if (ab == AB && nb == NB && kn == SB) return launch_rows_t<RowsCfg<AB, NB, SB>>(a, splits, part, s);
    FICCO_FOR_EACH_ROWS(X)
#undef X
    return FICCO_ERR_ARG;
}

// The few-rows kernel's tile, if it is expected to be faster than the other kernels' estimate (us); ab = 0: it is not. A CU draws the
// tile's rows and columns over all of k, at 146 KB a us alone and 90 when all do; a round of tiles more costs 2.5 us, since a
// CU holds one workgroup; and a launch cannot be faster than the weight's way through the chip, 7.3 TB/s if it is cached.
// Fitted to M 1-256 of eight shapes, K 512-16384, N 64-14336, each tile forced in turn (us, the other kernels / the tile taken:
// M 16, K 8192, N 3584 29.6 / 11.6; M 64 29.9 / 14.9; M 128 29.7 / 25.5; M 256 32.3, its best tile 48.9; M 64, K 4096, N 768 11.8 /
// 5.5; M 16, K 8192, N 64 18.8 / 5.9; M 64, K 4096, N 14336 21.6, its best tile 32.3). More rows pay where the columns are few, in one or
// two rounds: M 534, K 3584, N 432 14.0 / 8.9, M 1222, K 8896, N 192 33.2 / 22.4; not in three, M 1456, K 9856, N 432 41.5 / 68.3.
struct RowsTile {
    int ab, nb, splits;
};
RowsTile rows_tile(int64_t M, int64_t K, int64_t N, double us)
{
    RowsTile best{0, 0, 1};
    if (M > 2048) return best;
    const int cus = compute_units();
    auto consider = [&](int ab, int nb) {
        if (ab > 1 && M <= 8 * ab / 2) return;                 // half of the rows or more would not be there
        const int64_t tiles = ((M + 8 * ab - 1) / (8 * ab)) * ((N + 16 * nb - 1) / (16 * nb)), full = tiles / cus, rest = tiles - full * cus;
        if (tiles > (M > 512 ? 2 * cus : 0x7FFFFFFF / kRowsThreads)) return;       // ... or threads of a launch
        const double kb = (16 * nb + 8 * ab) * (double)K * 2e-3;
        const double drawn = (double)full * kb / 90 + (rest ? kb / (146.0 - 56.0 * (double)rest / cus) : 0) + 2.5 * (double)((tiles + cus - 1) / cus - 1);
        const double t = 3.0 + std::max(drawn, (double)(N * K + M * K) * 2 / 7.3e6);
        if (t < us * 0.999) { us = t; best = {ab, nb, 1}; }
    };
#define X(AB, NB, SB) if (!SB) consider(AB, NB);
    FICCO_FOR_EACH_ROWS(X)
#undef X
    return best;
}

// The same of a [K,N] weight, against the direct kernel (row_blocks, us: what that would take) or, row_blocks = 0, a tile's us. In one
// launch a workgroup has 32 columns, which puts twice as many CUs to work as 64; or k is split over as many workgroups of 64 columns
// (whole lines of the weight's rows) as make one round, and a second launch joins them. Which is the fastest depends on where the
// weight comes from: a CU draws 90-146 KB a us of it from the L2s (40-105 of half lines, the fewer the more CUs do), and from memory 43 (32). A loop over one
// layer finds a weight of up to 16 MiB in the L2s, a model's layers in turn do not; up to there the rule goes by the geometric mean
// of both. us, direct / one launch / splits (one layer | layers in turn): M 1, K 4096, N 768 9.0 / 6.5 / 9.0 | 14.5 / 15.8 / 10.3; M 64 of
// it 9.0 / 9.1 / 9.5 | 15.3 / 14.2 / 11.7; M 3, K 4800, N 560 10.0 / 7.0 / 9.0 | 20.5 / 17.2 / 11.2; beyond 16 MiB M 16, K 8192, N 3584
// - | 38 / 32 / 20; M 1, K 8192, N 1280 30 / 29 / 13; M 166, K 13184, N 264 50 / - / 19; M 32, K 16384, N 4096 68 / - / 42.
// Over the 110 random products (M to 500, K 1024-16384, N 64-6144) that the rates were fitted to, what it takes is 1.4 % slower than the fastest of
// these ways; the direct kernel or a tile throughout 42 %. Not in the estimates: that each of the row tiles reads the weight (eight times at M
// 64, where 8 and 16 rows a tile are estimated alike).
RowsTile rows_tile_kn(int64_t M, int64_t K, int64_t N, int row_blocks, double us)
{
    RowsTile best{0, 0, 1};
    if (M > 512) return best;
    const int cus = compute_units();
    const bool warm = K * N * 2 <= (16 << 20);
    auto both = [&](double in_l2, double from_memory) { return warm ? sqrt(in_l2 * std::max(in_l2, from_memory)) : from_memory; };
    if (row_blocks) {
        const int64_t tiles = ((M + 16 * row_blocks - 1) / (16 * row_blocks)) * ((N + 63) / 64);
        us = both(std::max(3.5, us - 2.5), 3.0 + (double)((tiles + cus - 1) / cus) * (16 * row_blocks + 64) * (double)K * 2e-3 / 43);
    }
    for (int ab = 1; ab <= 2; ++ab) {
        if (ab > 1 && M <= 8) break;
        for (int splits = 1; splits <= 16; splits *= 2) {
            const int nb = splits > 1 ? 4 : 2;
            const int64_t workgroups = ((M + 8 * ab - 1) / (8 * ab)) * ((N + 16 * nb - 1) / (16 * nb)) * splits;
            if (splits > 1 && K / kBK < splits * 8) break;             // a k-tile for each wavefront
            if (workgroups > cus) continue;
            const double kb = (16 * nb + 8 * ab) * (double)K * 2e-3 / splits;
            const double bytes = (double)(N * K + M * K) * 2 + (splits > 1 ? (double)splits * (double)(M * N) * 8 : 0);
            const double t = splits > 1 ? both(8.5 + kb / (146.0 - 56.0 * (double)workgroups / cus), 8.5 + std::max(kb / 43, bytes / 4.9e6))
                                        : both(3.0 + kb / (105.0 - 65.0 * (double)workgroups / cus), 5.0 + std::max(kb / 32, bytes / 4.9e6));
            if (t < us * (splits > 1 && best.splits == 1 ? 0.9 : 0.97)) { us = t; best = {ab, nb, splits}; }
        }
    }
    return best;
}

// ---------------------------------------------------------------------------------------------- turned operands, dZ
// src [R][Cc] (stride ld), 64 x 64 values a wavefront: a lane holds 8 rows x 8 columns, loads 16 bytes of each of 8 rows, turns
// the block with byte permutes and stores 16 bytes of each of 8 columns, so that loads and stores are whole 128-byte lines.
//   turned  [Cc][ldt], ldt = R rounded up to 64: src transposed, zero behind its end (null: not wanted)
//   with z (stride ldz): the value is src * act'(z), rounded to bf16, instead of src
//   same    [R][lds], lds = Cc rounded up to 64: the value in its own order, zero behind its end (null: not wanted)
//   sums    [ceil(R/64)][Cc] fp32: column sums over 64 rows each, of the values before they are rounded (null: not wanted)
// dZ is rounded to bf16 because the matrix instructions of its two products take bf16; with it dA and dW are off by 2.35e-3 of their
// 2-norm (M 8192, K 8192, N 3584 and M 1187, K 2880, N 1160 alike), of which 1.66e-3 are the rounding of the results themselves: a product of an
// unrounded dZ in two bf16 parts would be as near as that, at twice the matrix instructions (the large one 695 us of 755). dbias
// takes dZ as it is.
// Streaming, bound by memory: dZ of 8192 x 3584 in both orders 48 us, 4.9 TB/s. A workgroup is one wavefront, since small
// operands are then spread over more CUs; up to three operands go in one launch, the first with z.
struct TurnJob {
    const uint16_t *src, *z;
    uint16_t *turned, *same;
    float *sums;
    int64_t R, Cc, ld, ldz, ldt, lds;
};
struct TurnLaunch {
    TurnJob job[3];
    int32_t first[3];             // number of each job's first workgroup
};
constexpr int kTurnRows = 64;

// 16 bytes at `off` bytes from a uniform address, which stays in scalar registers
static __device__ __forceinline__ u32x4_t load_at(const uint16_t *base, uint32_t off)
{
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(reinterpret_cast<const char *>(base) + off));
}
static __device__ __forceinline__ void store_at(uint16_t *base, uint32_t off, u32x4_t v)
{
    *reinterpret_cast<u32x4_t *>(reinterpret_cast<char *>(base) + off) = v;
}

template <int ACT>
static __device__ __forceinline__ void turn_block(const TurnJob &a, int block)
{
    const int lane = threadIdx.x;
    // the wavefront's place, and the lane's in it
    const int tiles_c = (int)((a.Cc + 63) / 64), by = block / tiles_c;
    const int64_t R0 = (int64_t)by * kTurnRows, C0 = (int64_t)(block - by * tiles_c) * 64;
    const int lr = (lane & 7) * 8, lc = (lane >> 3) * 8;
    const int rows = (int)min((int64_t)64, a.R - R0), cols = (int)min((int64_t)64, a.Cc - C0);     // of the wavefront's, that exist
    const bool in = lc < cols;
    u32x4_t v[8];
    float sum[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) sum[c] = 0.f;
    {
        // rows and columns that are not there are read at the last that is, and then put to zero: a load under a condition of
        // its own makes the compiler copy all the others
        const uint16_t *src = a.src + R0 * a.ld + C0;
        const uint32_t c2 = (uint32_t)min(lc, cols - 8) * 2u;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = load_at(src, (uint32_t)min(lr + i, rows - 1) * ((uint32_t)a.ld * 2u) + c2);
        u32x4_t zz[8];
        if constexpr (ACT != FICCO_ACT_NONE) {
            const uint16_t *z = a.z + R0 * a.ldz + C0;
#pragma unroll
            for (int i = 0; i < 8; ++i) zz[i] = load_at(z, (uint32_t)min(lr + i, rows - 1) * ((uint32_t)a.ldz * 2u) + c2);
        }
        if (rows < 64 || cols < 64) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    v[i][p] = in && lr + i < rows ? v[i][p] : 0u;
                    if constexpr (ACT != FICCO_ACT_NONE) zz[i][p] = in && lr + i < rows ? zz[i][p] : 0u;
                }
        }
        if constexpr (ACT != FICCO_ACT_NONE) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const float lo = bf16_lo(v[i][p]) * slope<ACT>(bf16_lo(zz[i][p])), hi = bf16_hi(v[i][p]) * slope<ACT>(bf16_hi(zz[i][p]));
                    sum[2 * p] += lo;
                    sum[2 * p + 1] += hi;
                    v[i][p] = pack2_bf16_rne(lo, hi);
                }
        } else if (a.sums) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int p = 0; p < 4; ++p) { sum[2 * p] += bf16_lo(v[i][p]); sum[2 * p + 1] += bf16_hi(v[i][p]); }
        }
    }
    if (a.same && C0 + lc < a.lds) {
        uint16_t *same = a.same + R0 * a.lds + C0;
        const uint32_t off = ((uint32_t)lr * (uint32_t)a.lds + (uint32_t)lc) * 2u;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lr + i < rows) store_at(same + i * a.lds, off, v[i]);
    }
    if (a.turned && R0 + lr < a.ldt && in) {
        uint16_t *turned = a.turned + C0 * a.ldt + R0;
        const uint32_t off = ((uint32_t)lc * (uint32_t)a.ldt + (uint32_t)lr) * 2u;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            u32x4_t even, odd;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                even[i] = __builtin_amdgcn_perm(v[2 * i + 1][p], v[2 * i][p], 0x05040100u);
                odd[i] = __builtin_amdgcn_perm(v[2 * i + 1][p], v[2 * i][p], 0x07060302u);
            }
            store_at(turned + 2 * p * a.ldt, off, even);
            store_at(turned + (2 * p + 1) * a.ldt, off, odd);
        }
    }
    if (a.sums) {
        // over the 8 lanes of a column group
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] = lane_sum<8>(sum[c]);
        float t = sum[0];
#pragma unroll
        for (int c = 1; c < 8; ++c) t = (lane & 7) == c ? sum[c] : t;
        if (lane < cols) a.sums[(int64_t)by * a.Cc + C0 + lane] = t;
    }
}

template <int ACT>
__global__ __launch_bounds__(64) void turn_kernel(TurnLaunch a)
{
    const int block = blockIdx.x;
    if (block < a.first[1]) turn_block<ACT>(a.job[0], block);
    else if (block < a.first[2]) turn_block<FICCO_ACT_NONE>(a.job[1], block - a.first[1]);
    else turn_block<FICCO_ACT_NONE>(a.job[2], block - a.first[2]);
}

// Runs the jobs that have something to write, the first of them with the activation.
int launch_turn(int activation, TurnLaunch a, hipStream_t s)
{
    int64_t blocks = 0;
    for (int k = 0; k < 3; ++k) {
        TurnJob &j = a.job[k];
        a.first[k] = (int32_t)blocks;
        if (!j.turned && !j.same && !j.sums) continue;
        if (j.R < 1 || j.Cc < 8 || j.Cc % 8) return FICCO_ERR_SHAPE;
        blocks += ((j.R + kTurnRows - 1) / kTurnRows) * ((j.Cc + 63) / 64);
        if (blocks > 0x7FFFFFFF / 64) return FICCO_ERR_SHAPE;
    }
    if (!blocks) return FICCO_OK;
    const dim3 grid((unsigned)blocks), block(64);
    switch (activation) {
    case FICCO_ACT_NONE: hipLaunchKernelGGL(turn_kernel<FICCO_ACT_NONE>, grid, block, 0, s, a); break;
    case FICCO_ACT_RELU: hipLaunchKernelGGL(turn_kernel<FICCO_ACT_RELU>, grid, block, 0, s, a); break;
    case FICCO_ACT_GELU: hipLaunchKernelGGL(turn_kernel<FICCO_ACT_GELU>, grid, block, 0, s, a); break;
    case FICCO_ACT_GELU_TANH: hipLaunchKernelGGL(turn_kernel<FICCO_ACT_GELU_TANH>, grid, block, 0, s, a); break;
    case FICCO_ACT_SILU: hipLaunchKernelGGL(turn_kernel<FICCO_ACT_SILU>, grid, block, 0, s, a); break;
    default: return FICCO_ERR_ARG;
    }
    HIP_TRY(hipGetLastError());
    return FICCO_OK;
}

// out[c] = sum over r of in[r][c], r in [0, R). R = 0: zeros.
__global__ __launch_bounds__(1024) void sum_rows_kernel(const float *__restrict__ in, float *__restrict__ out, int R, int64_t Cc)
{
    __shared__ float s[32][32];
    const int64_t c = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
    const float t = column_sum(in + c, R, Cc, c < Cc, s);
    if (threadIdx.x < 32 && c < Cc) out[c] = t;
}

__global__ __launch_bounds__(256) void zero_kernel(u32x4_t *p, int64_t vecs)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < vecs; i += (int64_t)gridDim.x * 256) p[i] = u32x4_t{0u, 0u, 0u, 0u};
}

// ------------------------------------------------------------------------------------------------------------- host
// The struct with its defaults filled in; an error where it breaks a rule.
int checked(const ficco_linear_t *op, bool backward, ficco_linear_t *out)
{
    if (!op) return FICCO_ERR_ARG;
    ficco_linear_t o = *op;
    if (o.weight_layout < FICCO_WEIGHT_KN || o.weight_layout > FICCO_WEIGHT_NK || o.activation < FICCO_ACT_NONE || o.activation > FICCO_ACT_SILU ||
        o.bias_type < FICCO_BF16 || o.bias_type > FICCO_F32 || o.reserved)
        return FICCO_ERR_ARG;
    if (o.M < 0 || o.M > (backward ? kMaxK : 0x7FFFFFFF) || o.K < 1 || o.K % 64 || o.K > kMaxK || o.N < 1 || o.N % 8 || o.N > kMaxK) return FICCO_ERR_SHAPE;
    if (!o.lda) o.lda = o.K;
    if (!o.ldc) o.ldc = o.N;
    if (!o.ld_residual) o.ld_residual = o.N;
    if (!o.ld_pre) o.ld_pre = o.N;
    if (o.lda < o.K || o.lda % 8 || o.lda > kMaxK || o.ldc < o.N || o.ldc % 8 || o.ldc > kMaxK || o.ld_residual < o.N || o.ld_residual % 8 || o.ld_residual > kMaxK ||
        o.ld_pre < o.N || o.ld_pre % 8 || o.ld_pre > kMaxK)
        return FICCO_ERR_SHAPE;
    *out = o;
    return FICCO_OK;
}

// How a forward goes: row blocks of the direct kernel, for a small product of a [K,N] weight; or the few-rows kernel's tile; or the tile of
// the others, by the tile rule for operands in place. Whole tiles read a [K,N] weight as it is, but parts of tiles need it re-laid out. That
// copy is in no estimate (M 198, K 13440, N 2392 83 us a call with it, 53 of an [N,K] weight; M 465, K 14656, N 1112 74, 59).
struct Forward {
    int row_blocks, tile;
    RowsTile rows;
    int64_t bytes;
};
Forward choose_forward(int64_t M, int64_t K, int64_t N, bool kn)
{
    Forward f{};
    if (M == 0) return f;
    const Tile t = tile_for(M, K, N);
    double us = t.us;
    f.tile = t.id;
    if (kn) {
        // the direct kernel's offsets have 32 bits, and so has its launch's number of threads
        if (K * N * 2 <= 0x7FFFFFFF && (M + 15) / 16 * ((N + 63) / 64) <= 0x7FFFFFFF / 256) f.row_blocks = direct_row_blocks(M, K, N, compute_units(), us, &us);
        f.rows = rows_tile_kn(M, K, N, f.row_blocks, us);
        if (f.rows.ab) f.row_blocks = 0;
        else if (!f.row_blocks && !strided_tile(f.tile, false)) f.bytes = round_up(K * N * 2, 256);
    } else {
        f.rows = rows_tile(M, K, N, us);
    }
    if (f.rows.ab && f.rows.splits > 1) f.bytes = round_up(f.rows.splits * M * N * 4, 256);
    return f;
}

Forward forward_way(int64_t M, int64_t K, int64_t N, bool kn)
{
    return remembered<Forward>(M, K, N, kn, [&] { return choose_forward(M, K, N, kn); });
}

int run(const Forward &f, bool kn, LinearLaunch a, void *workspace, hipStream_t s)
{
    if (f.row_blocks) {
        DirectLaunch d{};
        d.A = a.A;
        d.W = a.W;
        d.C = a.C;
        d.M = a.M; d.N = a.N; d.K = a.K;
        HIP_TRY(launch_direct_epilogue(f.row_blocks, d, a.e, a.lda, a.ldc, s));
        return FICCO_OK;
    }
    if (f.rows.ab) return launch_rows(f.rows.ab, f.rows.nb, kn, a, f.rows.splits, (float *)workspace, s);
    if (kn && !f.bytes) return launch_tiles_strided(strided_tile(f.tile, false), false, a, s);
    if (kn) {
        HIP_TRY(launch_pack_weight(a.W, (uint16_t *)workspace, a.K, a.N, s));
        a.W = (const uint16_t *)workspace;
        a.ldw = a.K;
    }
    return launch_tiles(f.tile, a, s);
}

// How a backward goes, and the workspace, in bytes from its start (-1: not needed). dA is a forward product of dZ with W as a weight
// of the other layout. dW = A^T dZ has a tile of the kernel that reads A as it is (0: A is turned first).
struct Backward {
    int64_t Mp, Np;               // M and N rounded up to whole k-tiles
    Forward a;
    bool a_kn;
    int tile_w;
    int64_t dz, dz_turned, a_turned, w_other, part, sums, bytes;
};
Backward backward_way(const ficco_linear_t &o)
{
    Backward b{};
    b.Mp = round_up(o.M, kBK);
    b.Np = round_up(o.N, kBK);
    if (o.M == 0) return b;
    const bool kn = o.weight_layout == FICCO_WEIGHT_KN;
    // dA = dZ W^T sums over n, and an [N,K] weight has k next to each other; dW = A^T dZ sums over m, and A has k next to each other. What
    // lies behind the last n or m must be zero, which only a copy is.
    b.a_kn = !kn && b.Np == o.N;
    if (b.a_kn) {
        b.a = forward_way(o.M, b.Np, o.K, true);
        if (b.a.bytes && !b.a.rows.ab) b.a_kn = false;         // a copy: made with the others
    }
    if (!b.a_kn) b.a = forward_way(o.M, b.Np, o.K, false);
    if (b.Mp == o.M) b.tile_w = strided_tile(tile_for(kn ? o.K : o.N, b.Mp, kn ? o.N : o.K).id, kn);
    int64_t at = 0;
    auto take = [&](bool needed, int64_t bytes) {
        const int64_t here = at;
        if (needed) at += round_up(bytes, 256);
        return needed ? here : -1;
    };
    b.dz = take(o.activation != FICCO_ACT_NONE || b.Np != o.N, o.M * b.Np * 2);
    b.dz_turned = take(true, o.N * b.Mp * 2);
    b.a_turned = take(!b.tile_w, o.K * b.Mp * 2);
    b.w_other = take(!b.a_kn && (!kn || b.Np != o.N), o.K * b.Np * 2);
    b.part = take(b.a.bytes > 0, b.a.bytes);
    b.sums = take(true, (o.M + kTurnRows - 1) / kTurnRows * o.N * 4);
    b.bytes = at;
    return b;
}

// C[M,N] = A[M,K] B[N,K]^T with both operands k-contiguous and K a multiple of the k-tile.
int product(int64_t M, int64_t K, int64_t N, const uint16_t *A, int64_t lda, const uint16_t *B, uint16_t *C, hipStream_t s)
{
    GemmLaunch g{};
    g.A = A;
    g.Wt = B;
    g.C = C;
    g.lda = lda;
    g.ldc = N;
    g.N = (int32_t)N;
    g.K = (int32_t)K;
    g.n_blocks = 1;
    g.rows_per_block = (int32_t)M;
    HIP_TRY(launch_gemm(tile_for(M, K, N).id, g, s));
    return FICCO_OK;
}
// The same with A as [K][M] or B as [K][N].
int product_strided(int tile, bool a_strided, int64_t M, int64_t K, int64_t N, const uint16_t *A, int64_t lda, const uint16_t *B, int64_t ldb, uint16_t *C,
                    hipStream_t s)
{
    LinearLaunch l{};
    l.A = A;
    l.W = B;
    l.C = C;
    l.lda = lda;
    l.ldw = ldb;
    l.ldc = N;
    l.M = (int32_t)M;
    l.N = (int32_t)N;
    l.K = (int32_t)K;
    return launch_tiles_strided(tile, a_strided, l, s);
}

int zero(void *p, int64_t bytes, hipStream_t s)
{
    hipLaunchKernelGGL(zero_kernel, dim3((unsigned)std::min<int64_t>((bytes / 16 + 255) / 256, 1024)), dim3(256), 0, s, (u32x4_t *)p, bytes / 16);
    HIP_TRY(hipGetLastError());
    return FICCO_OK;
}

int sum_rows(const float *in, float *out, int64_t R, int64_t Cc, hipStream_t s)
{
    hipLaunchKernelGGL(sum_rows_kernel, dim3((unsigned)((Cc + 31) / 32)), dim3(1024), 0, s, in, out, (int)R, Cc);
    HIP_TRY(hipGetLastError());
    return FICCO_OK;
}

int forward(const ficco_linear_t *op, const void *A, const void *W, const void *bias, const void *residual, void *pre, void *C, void *workspace,
            int64_t workspace_bytes, hipStream_t s)
{
    ficco_linear_t o;
    int rc = checked(op, false, &o);
    if (rc) return rc;
    const bool none = o.M == 0;
    rc = check_args({{A, 16, none}, {W, 16, none}, {bias, o.bias_type == FICCO_F32 ? 4 : 2, true}, {residual, 16, true}, {pre, 16, true}, {C, 16, none}, {workspace, 16, true}});
    if (rc || none) return rc;
    const Forward f = forward_way(o.M, o.K, o.N, o.weight_layout == FICCO_WEIGHT_KN);
    if (f.bytes > 0 && (!workspace || workspace_bytes < f.bytes)) return FICCO_ERR_ARG;
    const Epilogue e{bias, (const uint16_t *)residual, (uint16_t *)pre, o.ld_residual, o.ld_pre, o.activation, o.bias_type == FICCO_F32};
    const bool kn = o.weight_layout == FICCO_WEIGHT_KN;
    return run(f, kn, LinearLaunch{(const uint16_t *)A, (const uint16_t *)W, (uint16_t *)C, o.lda, kn ? o.N : o.K, o.ldc, (int32_t)o.M, (int32_t)o.N, (int32_t)o.K, 0, e},
               workspace, s);
}

int backward(const ficco_linear_t *op, const void *A, const void *W, const void *pre, const void *dC, void *dA, void *dW, void *dbias, void *workspace,
             int64_t workspace_bytes, hipStream_t s)
{
    ficco_linear_t o;
    int rc = checked(op, true, &o);
    if (rc) return rc;
    const bool none = o.M == 0, act = o.activation != FICCO_ACT_NONE;
    rc = check_args({{A, 16, none || !dW}, {W, 16, none || !dA}, {pre, 16, none || !act}, {dC, 16, none}, {dA, 16, true}, {dW, 16, true}, {dbias, 4, true},
                     {workspace, 16, none}});
    if (rc) return rc;
    const int64_t M = o.M, K = o.K, N = o.N;
    if (none) {
        if (dW && (rc = zero(dW, K * N * 2, s))) return rc;
        return dbias ? sum_rows(nullptr, (float *)dbias, 0, N, s) : FICCO_OK;
    }
    const Backward b = backward_way(o);
    if (workspace_bytes < b.bytes) return FICCO_ERR_ARG;
    if (!dA && !dW && !dbias) return FICCO_OK;
    unsigned char *const ws = (unsigned char *)workspace;
    auto at = [&](int64_t off) { return off < 0 ? nullptr : (uint16_t *)(ws + off); };
    const bool kn = o.weight_layout == FICCO_WEIGHT_KN;

    // dZ as the products need it, with its column sums; A with m contiguous; W with n contiguous
    TurnLaunch t{};
    TurnJob &z = t.job[0], &ta = t.job[1], &tw = t.job[2];
    z.src = (const uint16_t *)dC;
    z.z = (const uint16_t *)pre;
    z.turned = dW ? at(b.dz_turned) : nullptr;
    z.same = dA ? at(b.dz) : nullptr;
    const bool one_block = M <= kTurnRows;                     // its sums are dbias
    z.sums = !dbias ? nullptr : one_block ? (float *)dbias : (float *)at(b.sums);
    z.R = M; z.Cc = N; z.ld = o.ldc; z.ldz = o.ld_pre; z.ldt = b.Mp; z.lds = b.Np;
    if (dW && !b.tile_w) {
        ta.src = (const uint16_t *)A;
        ta.turned = at(b.a_turned);
        ta.R = M; ta.Cc = K; ta.ld = o.lda; ta.ldt = b.Mp;
    }
    if (dA && b.w_other >= 0) {
        tw.src = (const uint16_t *)W;
        if (kn) { tw.same = at(b.w_other); tw.R = K; tw.Cc = N; tw.ld = N; tw.lds = b.Np; }
        else { tw.turned = at(b.w_other); tw.R = N; tw.Cc = K; tw.ld = K; tw.ldt = b.Np; }
    }
    if ((rc = launch_turn(o.activation, t, s))) return rc;
    if (dbias && !one_block && (rc = sum_rows(z.sums, (float *)dbias, (M + kTurnRows - 1) / kTurnRows, N, s))) return rc;
    const bool own = b.dz >= 0;
    const uint16_t *const dz = own ? at(b.dz) : (const uint16_t *)dC;
    const int64_t ldz = own ? b.Np : o.ldc;
    if (dA) {
        const uint16_t *const w = b.w_other >= 0 ? at(b.w_other) : (const uint16_t *)W;
        if (!b.a_kn && !b.a.rows.ab) rc = product(M, b.Np, K, dz, ldz, w, (uint16_t *)dA, s);
        else rc = run(b.a, b.a_kn, LinearLaunch{dz, w, (uint16_t *)dA, ldz, b.a_kn ? K : b.Np, K, (int32_t)M, (int32_t)K, (int32_t)b.Np, 0, {}}, at(b.part), s);
        if (rc) return rc;
    }
    if (dW) {
        // in the order that gives dW W's layout
        const uint16_t *const a = (const uint16_t *)A, *const zt = at(b.dz_turned);
        if (b.tile_w && kn) rc = product_strided(b.tile_w, true, K, M, N, a, o.lda, zt, M, (uint16_t *)dW, s);
        else if (b.tile_w) rc = product_strided(b.tile_w, false, N, M, K, zt, M, a, o.lda, (uint16_t *)dW, s);
        else if (kn) rc = product(K, b.Mp, N, at(b.a_turned), b.Mp, zt, (uint16_t *)dW, s);
        else rc = product(N, b.Mp, K, zt, b.Mp, at(b.a_turned), (uint16_t *)dW, s);
        if (rc) return rc;
    }
    return FICCO_OK;
}

}  // namespace
}  // namespace ficco

using namespace ficco;

extern "C" {

int ficco_linear_workspace(const ficco_linear_t *op, int backward, int64_t *bytes)
{
    return guarded([&] {
        ficco_linear_t o;
        if (!bytes) return (int)FICCO_ERR_ARG;
        const int rc = checked(op, backward != 0, &o);
        if (rc) return rc;
        *bytes = backward ? backward_way(o).bytes : forward_way(o.M, o.K, o.N, o.weight_layout == FICCO_WEIGHT_KN).bytes;
        return (int)FICCO_OK;
    });
}

int ficco_linear(const ficco_linear_t *op, const void *A, const void *W, const void *bias, const void *residual, void *pre, void *C, void *workspace,
                 int64_t workspace_bytes, void *stream)
{
    return guarded([&] { return forward(op, A, W, bias, residual, pre, C, workspace, workspace_bytes, (hipStream_t)stream); });
}

int ficco_linear_backward(const ficco_linear_t *op, const void *A, const void *W, const void *pre, const void *dC, void *dA, void *dW, void *dbias,
                          void *workspace, int64_t workspace_bytes, void *stream)
{
    return guarded([&] { return backward(op, A, W, pre, dC, dA, dW, dbias, workspace, workspace_bytes, (hipStream_t)stream); });
}

}  // extern "C"

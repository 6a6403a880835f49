// The linear operator's product over tiles (see ficco_linear.hip): the kernel and its launch, for the files that instantiate it. Not
// installed.
#pragma once
#include "ficco_operators.h"
#include "ficco_epilogue.h"

namespace ficco {

// C[M,N] from A and W, whose k values lie next to each other (A [M][K] with row stride lda, W [N][K] with ldw) or not (A [K][M],
// W [K][N]; M and N multiples of 8 then); K a multiple of the k-tile.
struct LinearLaunch {
    const uint16_t *A, *W;
    uint16_t *C;
    int64_t lda, ldw, ldc;
    int32_t M, N, K, group_m;
    Epilogue e;
};

// One launch over all tiles, at most as many workgroups as run at once; the tiles in the order of gemm_blocks_kernel. M 16384, K 8192,
// N 3584 with GELU and its argument stored: 730 us, 1.32 PFLOP/s, at the card's power limit; a large library product reaches 1.4-1.5.
// SA, SB: A, W as [K][...]. Not both: the transposing reads move 64 bytes a cycle where the others move 128, and with both operands
// through them LDS is what the kernel waits for (dW of M 8192, K 8192, N 3584 390 us; one of them 345, none 333).
template <class T, bool SA, bool SB>
__global__ __launch_bounds__(T::THREADS) void linear_tiles_kernel(LinearLaunch a)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int tiles_n = (a.N + T::BN - 1) / T::BN;
    const int tiles_m = (int)(((int64_t)a.M + T::BM - 1) / T::BM);
    const XcdRun run = xcd_run(blockIdx.x, gridDim.x, tiles_m * tiles_n);
    const int per_group = a.group_m * tiles_n;
    for (int t = run.first; t < run.count; t += run.stride) {
        const int lid = run.start + t;
        const int group = lid / per_group;
        const int first_m = group * a.group_m;
        const int gsz = min(tiles_m - first_m, a.group_m);
        const int tm = first_m + (lid % per_group) % gsz;
        const int tn = (lid % per_group) / gsz;
        const int64_t row0 = (int64_t)tm * T::BM;
        const int rows_valid = (int)min((int64_t)T::BM, a.M - row0);
        const int col0 = tn * T::BN;
        const int cols_valid = min(T::BN, a.N - col0);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
        const uint16_t *const w = SB ? a.W + col0 : a.W + (int64_t)col0 * a.ldw;
        TileAcc<T> ta;
        tile_zero(ta);
        if constexpr (SA) {
            StridedA<T> pa(a.A + row0, rows_valid, a.lda, wave, lane);
            tile_accumulate_from<T, NoHook, StridedA<T>, KStrided, KContiguous>(ta, pa, w, cols_valid, a.ldw, a.K, smem);
        } else {
            typedef std::conditional_t<SB, KStrided, KContiguous> LayB;
            PlainA<T> pa(a.A + row0 * a.lda, rows_valid, a.lda, wave, lane);
            tile_accumulate_from<T, NoHook, PlainA<T>, KContiguous, LayB>(ta, pa, w, cols_valid, a.ldw, a.K, smem);
        }
        with_activation(a.e.activation, [&](auto act) __attribute__((always_inline)) {
            tile_store_epilogue<T, act.value>(ta, a.e, a.C + row0 * a.ldc + col0, rows_valid, cols_valid, a.ldc, row0, col0);
        });
        __syncthreads();                   // everyone is done with the ring before the next tile refills it
    }
    wait_vmem<0>();                        // no load may arrive in LDS that is not this workgroup's any more
}

template <class T, bool SA, bool SB>
int launch_tiles_t(const LinearLaunch &a, hipStream_t s)
{
    const int64_t tiles_n = ((int64_t)a.N + T::BN - 1) / T::BN, tiles_m = ((int64_t)a.M + T::BM - 1) / T::BM, total = tiles_m * tiles_n;
    if (total <= 0 || total > 0x7FFFFFFF || a.lda > kMaxK || a.ldw > kMaxK || a.K < kBK || a.K % kBK) return FICCO_ERR_SHAPE;
    static_assert(!(SA && SB), "one of the two");
    if ((SA && a.M % 8) || a.N % 8) return FICCO_ERR_SHAPE;
    static int fit_of[64];                 // per device: workgroups that run at once, 0 = not asked yet
    int dev = 0;
    HIP_TRY(hipGetDevice(&dev));
    int fit = dev < 64 ? fit_of[dev] : 0;
    if (fit == 0) {
        const auto fn = &linear_tiles_kernel<T, SA, SB>;
        int per_cu = 0;
        HIP_TRY((raise_lds_limit<&linear_tiles_kernel<T, SA, SB>>(T::LDS_BYTES)));
        HIP_TRY(hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, fn, T::THREADS, T::LDS_BYTES));
        fit = std::max(8, per_cu * compute_units() / 8 * 8);
        if (dev < 64) fit_of[dev] = fit;
    }
    const int64_t grid = std::min<int64_t>(total, fit);
    LinearLaunch b = a;
    b.group_m = 8;
    if (total > grid) {
        double best = -1;
        for (int g = 1; g <= 8; g *= 2) {
            const double c = tile_order_cost(T::BM, T::BN, tiles_n, tiles_m, grid / 8, 1, g, (int64_t)a.M * a.K * 2, (int64_t)a.N * a.K * 2);
            if (best < 0 || c < best) { best = c; b.group_m = g; }
        }
    }
    hipLaunchKernelGGL((linear_tiles_kernel<T, SA, SB>), dim3((unsigned)grid), dim3(T::THREADS), T::LDS_BYTES, s, b);
    HIP_TRY(hipGetLastError());
    return FICCO_OK;
}

// ficco_linear_strided.hip: with A (a_strided) or W not k-contiguous. Parts of tiles have no such form, nor do tiles of 32 rows with
// such an A (rows of 64 bytes): strided_tile() = the tile to take instead of the tile rule's, 0 = none.
int launch_tiles_strided(int tile, bool a_strided, const LinearLaunch &a, hipStream_t s);
inline int strided_tile(int tile, bool a_strided) { return is_part(tile) ? 0 : a_strided && tile == TILE_32x256 ? TILE_64x256 : tile; }

}  // namespace ficco

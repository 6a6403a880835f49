// The tile routine that the GEMM kernels share: zero, accumulate over a k range, store. See ficco_gemm.hip for the data flow and
// what bounds it. Not installed.
#pragma once
#include "ficco_internal.h"
#include "ficco_mfma.h"

namespace ficco {

// A workgroup tile and the schedule of its k loop. The loop's unit is the slot: one v_mfma_f32_16x16x32_bf16 and what
// is issued behind it. A turn of TT slots multiplies one k-tile (a stage of 64 k values, two halves of 32); see
// tile_accumulate_from for what the positions mean.
template <int BM_, int BN_, int WGM_, int WGN_, int NSTAGE_>
struct TileCfg {
    static constexpr int BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_;
    static constexpr int NSTAGE = NSTAGE_;                     // LDS stages in the ring: the loads of k-tile k + NSTAGE follow the reads of k-tile k
    static constexpr int BK = kBK;
    static constexpr int ROWB = BK * 2;                        // bytes of a row of a stage
    static constexpr int SLOTS = BK / 8;                       // 16-byte slots per row
    static constexpr int RPL = 1024 / ROWB;                    // rows one load instruction (64 lanes x 16 B) fills
    static constexpr int THREADS = WGM * WGN * 64;
    static constexpr int WTM = BM / WGM, WTN = BN / WGN;       // wavefront tile
    static constexpr int FM = WTM / 16, FN = WTN / 16;         // 16x16 MFMA blocks per wavefront
    static constexpr int A_STAGE = BM * ROWB, B_STAGE = BN * ROWB;   // bytes
    static constexpr int STAGE = A_STAGE + B_STAGE;
    static constexpr int LDS_BYTES = NSTAGE * STAGE;
    static constexpr int NW = WGM * WGN;                       // wavefronts, one per SIMD
    static constexpr int AB = BM / RPL / NW, BB = BN / RPL / NW; // 1 KiB blocks loaded per wavefront per stage
    static constexpr int LOADS = AB + BB;                      // load instructions per wavefront per k-tile
    static constexpr int NM = FM * FN, TT = 2 * NM;            // MFMAs per half and per turn
    static constexpr int NR = FM + FN;                         // fragment reads per half
    // LDS hands a wavefront one 1 KiB fragment in about 32 cycles when all four read: a read every second slot where the
    // turn has the slots for it.
    static constexpr int RSTEP = TT >= 4 * NR ? 2 : 1;
    // Two stages: the stage is free (FREE) long before the other one is needed (LAND). More stages: one barrier does both.
    static constexpr bool SPLIT = NSTAGE == 2 && TT >= 64;
    static constexpr int R1 = SPLIT ? 6 : 0;                   // first slot of the reads of this k-tile's second half
    static constexpr int FREE = R1 + NR * RSTEP + (SPLIT ? 2 : RSTEP == 2 ? 4 : 3);
    static constexpr int LAND = SPLIT ? TT + 4 - 2 * (NR - 1) - 2 : FREE;
    static constexpr int R0 = SPLIT ? LAND + 2 : LAND + 1;     // first slot of the reads of the next k-tile's first half
    static constexpr int LS = FREE + 1;                        // first load of k-tile k + NSTAGE
    static constexpr int LSTEP = NSTAGE == 2 && !SPLIT ? 2 : TT / LOADS > 0 ? TT / LOADS : 1;
    static constexpr bool at(int dist, int step, int count) { return dist >= 0 && dist % step == 0 && dist / step < count; }
    static constexpr int load_slot(int l) { return LS + l * LSTEP; }
    static constexpr int loads_before(int slot) { int n = 0; for (int l = 0; l < LOADS; ++l) n += load_slot(l) < slot; return n; }
    static constexpr int WRAPPED = LOADS - loads_before(TT);   // loads that fall into the next turn
    // loads in flight at LAND that are younger than those of the next k-tile
    static constexpr int younger_at_land() { int n = 0; for (int e = 0; e + 2 <= NSTAGE; ++e) n += loads_before(LAND + e * TT); return n; }
    // First and last slot of a half whose MFMA uses fragment q (row block 0, the column blocks, the other row blocks; column
    // blocks go back and forth from row block to row block).
    static constexpr int first_use(int q) { return q == 0 ? 0 : q <= FN ? q - 1 : (q - FN) * FN; }
    static constexpr int last_use(int q)
    {
        return q == 0 ? FN - 1 : q <= FN ? (FM - 1) * FN + (FM % 2 ? q - 1 : FN - q) : (q - FN) * FN + FN - 1;
    }
    // A half's fragments are replaced behind their last MFMA and there before their first. (256x128 and 128x256 begin to
    // read the next k-tile's first half three MFMAs before this one's is done with.)
    static constexpr bool fragments_hold()
    {
        for (int q = 0; q < NR; ++q) {
            const int r0 = R0 + q * RSTEP, r1 = R1 + q * RSTEP;
            if (r0 < last_use(q) || (r0 >= TT && r0 - TT >= first_use(q)) || r1 >= NM + first_use(q)) return false;
        }
        return true;
    }
    // Stages go in pairs (tile_accumulate_burst).
    static constexpr bool BURST = NM <= 4;
    static_assert(BURST || fragments_hold(), "a fragment is read too early or too late");
    static_assert(BURST ? NSTAGE % 2 == 0 && NSTAGE >= 6 && (NSTAGE - 2) * LOADS < 64 : NSTAGE >= 2 && NSTAGE <= 6 && (NSTAGE - 1) * LOADS < 64,
                  "ring of 2 to 6 stages, or pairs of them, vmcnt has 6 bits");
    static_assert(LDS_BYTES <= 160 * 1024 - 64, "LDS ring plus the kernels' few static words must fit one CU");
    static_assert(THREADS == 256, "4 wavefronts");
    static_assert(BM % (RPL * NW) == 0 && BN % (RPL * NW) == 0, "every wavefront loads the same number of blocks");
    static_assert(WTM % 16 == 0 && WTN % 32 == 0, "wavefront tile is made of 16x16 blocks, stored in pairs along a row");
    static_assert(AB >= 1 && BB >= 1, "tile too small for the loader");
    static_assert(BURST || (R0 + (NR - 1) * RSTEP - TT < (FM - 1) * FN && R0 + (NR - 1) * RSTEP - TT < FREE && load_slot(LOADS - 1) - TT < LS && load_slot(LOADS - 1) < LAND + (NSTAGE - 1) * TT),
                  "what a turn leaves to the next one is done before it is needed");
};

// Computes one BM x BN tile. a_tile: first row of the tile in A; rows_valid in [1, BM] rows of
// it exist (the others are neither stored nor allowed to fault: their loads are clamped to the
// last valid row). wt_tile: first row (= output column) of the tile in Wt; cols_valid likewise.
//
// LDS holds a ring of NSTAGE stages; a stage is BM + BN rows of 128 B (64 k values), the 16-byte
// slot kc of row r stored at slot kc ^ ((r >> 1) & 7) so that the 16 lanes of a ds_read_b128 phase
// hit 64 different banks. Loads go global -> LDS directly (no staging registers): a wavefront
// instruction fills 8 rows, lane l fetching the slot that belongs at position l. The big tile only
// has room for two stages; the smaller tiles use three or four, which is what keeps launches with
// few workgroups (small pieces) from being bound by load latency. The loop itself is described in
// tile_accumulate_from.
template <class T>
struct TileAcc {
    f32x4_t acc[T::FN][T::FM];
};

template <class T>
static __device__ __forceinline__ void tile_zero(TileAcc<T> &ta)
{
#pragma unroll
    for (int j = 0; j < T::FN; ++j)
#pragma unroll
        for (int i = 0; i < T::FM; ++i) ta.acc[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // the MFMAs are inline assembly, so the compiler does not know what they need after a write to their accumulators
    asm volatile("s_nop 7" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

struct NoHook {
    __device__ __forceinline__ void operator()() const {}
};

// Byte offset, from the first row of the tile, of what lane `lane` fetches for 1 KiB block `blk` of a stage:
// row blk*RPL + lane/SLOTS (clamped to the last row that exists), 16-byte slot (lane%SLOTS) ^ swizzle(row) of
// its k-tile. The swizzle - (row>>1)&7, two rows of 128 B share a 256-byte line of banks - spreads the rows over
// different slots, so that the 16 lanes of a ds_read_b128 phase, which read one k slot of 16 consecutive rows, hit 64
// different banks.
template <class T>
static __device__ __forceinline__ uint32_t lane_offset(int blk, int lane, int rows_valid, int64_t row_stride_elems)
{
    const int row = blk * T::RPL + lane / T::SLOTS;
    const int kc = (lane % T::SLOTS) ^ ((row >> 1) & (T::SLOTS - 1));
    const int rr = row < rows_valid ? row : rows_valid - 1;
    return (uint32_t)(((int64_t)rr * row_stride_elems + kc * 8) * 2);
}

// Where the loader finds its part of k-tile kt of A. PlainA: one row-major block [rows, K] with row stride lda:
// a wave-uniform base that moves along k, and one per-lane byte offset per load (the tile's rows must span less
// than 4 GiB, which the shape rules guarantee: at most 256 rows of at most 2^31 elements... of 2 bytes - the
// launchers refuse row strides above kMaxK).
template <class T>
struct PlainA {
    uint32_t off[T::AB];
    const uint16_t *base;
    __device__ __forceinline__ PlainA(const uint16_t *a_tile, int rows_valid, int64_t lda, int wave, int lane) : base(scalar_base(a_tile))
    {
#pragma unroll
        for (int i = 0; i < T::AB; ++i) off[i] = lane_offset<T>(wave * T::AB + i, lane, rows_valid, lda);
    }
    __device__ __forceinline__ void seek(int) {}
    __device__ __forceinline__ const uint16_t *at(int kt) const { return base + (int64_t)kt * T::BK; }
};

// SlicedA: a run of consecutive k slices of the K-sliced layout (slice s = the [M][k0[s+1]-k0[s]] block that
// starts at element M*k0[s]), read as one k range. The issue stream walks the k-tiles in ascending order;
// `seek` moves to the slice a k-tile lies in and only then rebuilds the base and the per-lane offsets for that
// slice's row stride, so that inside a slice a load costs what it costs with PlainA.
template <class T>
struct SlicedA {
    uint32_t off[T::AB];
    const uint16_t *base;
    const uint16_t *A;
    const int32_t *k0;
    int64_t M, row0;
    int sl, kt_begin, kt_end, rows_valid, wave, lane;
    __device__ __forceinline__ SlicedA(const uint16_t *A_, const int32_t *k0_, int64_t M_, int64_t row0_, int first_slice, int rows_valid_,
                                       int wave_, int lane_)
        : base(A_), A(A_), k0(k0_), M(M_), row0(row0_), sl(first_slice - 1), kt_begin(0), kt_end(0), rows_valid(rows_valid_), wave(wave_), lane(lane_)
    {
    }
    __device__ __forceinline__ void seek(int kt)
    {
        while (kt >= kt_end) {               // uniform: every lane takes the same steps
            ++sl;
            const int kb = scalar(k0[sl]), kw = scalar(k0[sl + 1]) - kb;
            kt_begin = kt_end;
            kt_end += kw / T::BK;
            base = scalar_base(A + M * kb + row0 * kw);
#pragma unroll
            for (int i = 0; i < T::AB; ++i) off[i] = lane_offset<T>(wave * T::AB + i, lane, rows_valid, kw);
        }
    }
    __device__ __forceinline__ const uint16_t *at(int kt) const { return base + (int64_t)(kt - kt_begin) * T::BK; }
};

// How an operand lies in memory: a row's k values next to each other (KContiguous), or a k value's rows next to each other
// (KStrided: the operand as [k][DIM], row stride ld, as the caller has it where the other layout would be a copy). A stage of the
// latter is 64 rows of 2 DIM bytes, a fragment comes out of it by transposing reads (ds_read_b64_tr_b16: 16 lanes read 4 rows
// x 16 columns, lane i gets column i; two of them make a fragment's 8 k values). 16-byte slot s of row r lies at s ^
// strided_swizzle(r): half a wavefront's transposing read touches rows 0-3 and 8-11, 32 bytes each, which this spreads over all
// 64 banks (rows that are multiples of 256 bytes need all 8 places of it, others differ by half of it already).
struct KContiguous { static constexpr bool STRIDED = false; };
struct KStrided { static constexpr bool STRIDED = true; };
template <int DIM>
static __device__ __forceinline__ int strided_swizzle(int row)
{
    static_assert(DIM % 64 == 0 || DIM == 32, "whole lines, or halves of them");
    if constexpr (DIM == 32) return 2 * ((row >> 3) & 1);      // four rows fill the banks
    return DIM % 128 == 0 ? 2 * ((row & 3) | (((row >> 3) & 1) << 2)) : 2 * (((row >> 1) & 1) | (((row >> 3) & 1) << 1));
}
// Byte offset, from the tile's first column of its first row, of what lane `lane` fetches for 1 KiB block `blk` of a stage (columns
// that are not there: the last eight that are; `valid` is a multiple of 8)
template <int DIM>
static __device__ __forceinline__ uint32_t strided_lane_offset(int blk, int lane, int valid, int64_t ld)
{
    constexpr int SLOTS = DIM / 8;
    const int at = blk * 64 + lane, row = at / SLOTS, slot = (at % SLOTS) ^ strided_swizzle<DIM>(row);
    return (uint32_t)(((int64_t)row * ld + min(slot, valid / 8 - 1) * 8) * 2);
}
// A of a KStrided operand: see PlainA
template <class T>
struct StridedA {
    uint32_t off[T::AB];
    const uint16_t *base;
    int64_t step;
    __device__ __forceinline__ StridedA(const uint16_t *a_tile, int rows_valid, int64_t lda, int wave, int lane) : base(scalar_base(a_tile)), step(lda * T::BK)
    {
#pragma unroll
        for (int i = 0; i < T::AB; ++i) off[i] = strided_lane_offset<T::BM>(wave * T::AB + i, lane, rows_valid, lda);
    }
    __device__ __forceinline__ void seek(int) {}
    __device__ __forceinline__ const uint16_t *at(int kt) const { return base + kt * step; }
};
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4_t;
// A fragment (16 rows of the operand, 32 k values) out of a KStrided stage: addr = LDS address of the lane's part
template <int DIM>
static __device__ __forceinline__ bf16x8_t strided_fragment(uint32_t addr)
{
    union { i16x4_t h[2]; bf16x8_t v; } n;
    n.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t *)(uintptr_t)addr);
    n.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t *)(uintptr_t)(addr + 4 * DIM * 2));
    return n.v;
}

// One MFMA: 16 columns of the packed weight x 16 rows of A x 32 k. The operands are passed swapped (D[n][m]), so that
// a lane ends up with 4 consecutive columns of one C row. Inline assembly with the accumulator tied to the
// accumulation registers: the builtin leaves the register allocator free to move the 256 of the big tile between the
// two halves of the register file, which it does with hundreds of copies per turn.
static __device__ __forceinline__ void mfma_16x16x32(f32x4_t &c, const bf16x8_t &n, const bf16x8_t &m)
{
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(n), "v"(m));
}

// The k loop of tiles whose turn has too few MFMAs to put anything behind. A turn is two stages (128 k values): one wait and
// one barrier, behind which its k-tiles have landed for everyone and everyone has read the two before; then all of its
// fragments out of LDS; then the loads that refill the two stages before it, with the MFMAs between them, as their fragments
// arrive (a wavefront's loads take 64 cycles each while all four issue theirs, and what is behind a load waits for that).
//
// What bounds it: the CU draws 64 bytes a cycle from L2 and 45-52 from beyond, whatever is in flight. 32x64 tiles draw 24 KiB
// a turn, 64x64 32 KiB, where 64x128 draws 48: 0.26 / 0.35 / 0.45 us, of which the loads alone are 0.22 / 0.31 / 0.45. MFMAs
// behind all loads 0.275 / 0.41; touching the lines a few turns ahead with a fifth wavefront 0.42 / 0.52, because a touched
// line takes the same way.
template <class T, class Hook, class AddrA>
static __device__ __forceinline__ void tile_accumulate_burst(TileAcc<T> &ta, AddrA &pa, const uint16_t *__restrict__ wt_tile, int cols_valid,
                                                             int64_t ldw, int K, unsigned char *smem, Hook after_first_wait)
{
    const int lane = threadIdx.x & 63;
    const int wave = scalar(threadIdx.x >> 6);
    const int wm = wave / T::WGN, wn = wave % T::WGN;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    const uint16_t *const wt = scalar_base(wt_tile);
    constexpr int TURNS = T::NSTAGE / 2, PAIR = 2 * T::STAGE, LOADS = 2 * T::LOADS;
    const int KT = scalar(K) / T::BK, KP = (KT + 1) / 2;
    uint32_t offb[T::BB];
#pragma unroll
    for (int i = 0; i < T::BB; ++i) offb[i] = lane_offset<T>(wave * T::BB + i, lane, cols_valid, ldw);
    // load l of a turn's: those of its first k-tile, then those of its second (which may not exist at the end of K: the first
    // again, and not used)
    auto load = [&](int t, uint32_t pair, auto l_c) __attribute__((always_inline)) {
        constexpr int u = decltype(l_c)::value / T::LOADS, l = decltype(l_c)::value % T::LOADS;
        const int kt = min(2 * t + u, KT - 1);
        if constexpr (l == 0) pa.seek(kt);
        if constexpr (l < T::AB) set_lds_target<u * T::STAGE + l * 1024>(lds0 + pair + wave * T::AB * 1024);
        else set_lds_target<u * T::STAGE + T::A_STAGE + (l - T::AB) * 1024>(lds0 + pair + wave * T::BB * 1024);
        asm volatile("s_nop 0" ::: "memory");
        if constexpr (l < T::AB) load_to_lds_16(pa.at(kt), pa.off[l]);
        else load_to_lds_16(wt + (int64_t)kt * T::BK, offb[l - T::AB]);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto issue = [&](int t, uint32_t pair) __attribute__((always_inline)) {
        static_for<LOADS>([&](auto l) __attribute__((always_inline)) { load(t, pair, l); });
    };
    const int frow = lane & 15, fh = lane >> 4, fs = (frow >> 1) & 7;
    const int a_base = (wm * T::WTM + frow) * T::ROWB, b_base = T::A_STAGE + (wn * T::WTN + frow) * T::ROWB;
    bf16x8_t fa[4][T::FM], fb[4][T::FN];
    auto read = [&](uint32_t pair) __attribute__((always_inline)) {
        static_for<4>([&](auto h_c) __attribute__((always_inline)) {
            constexpr int h = decltype(h_c)::value;
            const unsigned char *base = smem + pair + h / 2 * T::STAGE + (((4 * (h % 2) + fh) ^ fs) << 4);
#pragma unroll
            for (int i = 0; i < T::FM; ++i) fa[h][i] = *reinterpret_cast<const bf16x8_t *>(base + a_base + i * 16 * T::ROWB);
#pragma unroll
            for (int j = 0; j < T::FN; ++j) fb[h][j] = *reinterpret_cast<const bf16x8_t *>(base + b_base + j * 16 * T::ROWB);
        });
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int NMF = 4 * T::NM;         // MFMAs of a turn
    auto product = [&](auto m_c) __attribute__((always_inline)) {
        constexpr int m = decltype(m_c)::value, h = m / T::NM, i = m % T::NM / T::FN, j = m % T::FN;
        mfma_16x16x32(ta.acc[j][i], fb[h][j], fa[h][i]);
    };
    auto meet = [&](auto in_flight) __attribute__((always_inline)) {
        wait_vmem<decltype(in_flight)::value>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wg_barrier();
    };
    const int ahead = min(KP, TURNS - 1);
    for (int t = 0; t < ahead; ++t) issue(t, t * PAIR);
    uint32_t cur = 0, next = (TURNS - 1) * PAIR;
    int k = 0;
#pragma clang loop unroll(disable)
    for (; k + TURNS - 1 < KP; ++k) {
        meet(std::integral_constant<int, (TURNS - 2) * LOADS>{});
        if (k == 0) after_first_wait();
        read(cur);
        static_for<LOADS>([&](auto l) __attribute__((always_inline)) {
            load(k + TURNS - 1, next, l);
            static_for<NMF>([&](auto m) __attribute__((always_inline)) {
                if constexpr (l.value == 1 + m.value * (LOADS - 1) / NMF) product(m);
            });
            __builtin_amdgcn_sched_barrier(0);
        });
        cur = cur == (TURNS - 1) * PAIR ? 0 : cur + PAIR;
        next = next == (TURNS - 1) * PAIR ? 0 : next + PAIR;
    }
    static_for<TURNS - 1>([&](auto t) __attribute__((always_inline)) {
        constexpr int left = TURNS - 1 - decltype(t)::value;
        if (left <= ahead) {
            meet(std::integral_constant<int, (left - 1) * LOADS>{});
            if (k == 0) after_first_wait();
            read(cur);
            static_for<NMF / 2>([&](auto m) __attribute__((always_inline)) { product(m); });
            if (2 * k + 1 < KT) static_for<NMF / 2>([&](auto m) __attribute__((always_inline)) { product(std::integral_constant<int, NMF / 2 + m.value>{}); });
            ++k;
            cur = cur == (TURNS - 1) * PAIR ? 0 : cur + PAIR;
        }
    });
    // accumulators may be read after the last MFMA's passes
    asm volatile("s_nop 15" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The k loop. Turn k multiplies k-tile k out of registers: slots [0, NM) its first half (k values 0..31 of the stage),
// whose fragments were read during the turn before, slots [NM, TT) its second half, whose fragments are read during
// the first (from slot R1 on). Behind the MFMAs go, at fixed slots (TileCfg),
//   FREE   all of this wavefront's reads of the stage are in registers; barrier: that holds for every wavefront
//   LS...  the loads of k-tile k + NSTAGE into the stage just freed, one every LSTEP slots, spread over a whole turn:
//          the last WRAPPED of them fall into turn k + 1
//   LAND   k-tile k + 1 has landed for this wavefront's loads; barrier: for everyone's
//   R0...  the reads of the first half of k-tile k + 1
// so that no wait ever has an MFMA's operands behind it, a load has between half a turn and a turn and a half (two
// stages) to arrive, and the address path, which takes 16 cycles per load and is shared by the four wavefronts, sees
// them evenly. All issue order is pinned (sched_barrier); what the compiler adds are the LDS waits of the fragments.
//
// What it measured on the 256x256 tile (M 4096, K 16384, N 4096: one round of tiles; random data, board at its 1400 W):
// v_mfma_f32_32x32x16 in this loop 1326 TFLOP/s, v_mfma_f32_16x16x32 1399 (half the accumulator traffic per flop, and
// the same bits); its loads spread over the turn instead of one every four slots 1512 (a denser issue holds up the
// MFMAs behind it); M0 written a slot ahead of its load 1552; this loop's row-segment stores 1556. The loop before it
// (32x32x16, one barrier per turn, the loads of a k-tile within half a turn) 1244; the vendor library 1596-1650.
// Counters (M 16384, K 8192, N 3584): 2446 cycles a turn, epilogues included, of which 2048 are MFMAs.
template <class T, class Hook = NoHook, class AddrA = PlainA<T>, class LayA = KContiguous, class LayB = KContiguous>
static __device__ __forceinline__ void tile_accumulate_from(TileAcc<T> &ta, AddrA &pa,
                                                            const uint16_t *__restrict__ wt_tile, int cols_valid,
                                                            int64_t ldw, int K, unsigned char *smem,
                                                            Hook after_first_wait = Hook())
{
    static_assert(!T::BURST || (!LayA::STRIDED && !LayB::STRIDED), "the paired loop reads k-contiguous operands");
    if constexpr (T::BURST) {
        tile_accumulate_burst<T, Hook, AddrA>(ta, pa, wt_tile, cols_valid, ldw, K, smem, after_first_wait);
        return;
    } else {
    f32x4_t (&acc)[T::FN][T::FM] = ta.acc;
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / T::WGN, wn = wave % T::WGN;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    const uint16_t *const wt = scalar_base(wt_tile);
    constexpr int D = T::NSTAGE;           // k-tiles between a stage's reads and the loads that refill it

    uint32_t offb[T::BB];                  // per-lane byte offsets of the W loads from the tile's first row
#pragma unroll
    for (int i = 0; i < T::BB; ++i) {
        if constexpr (LayB::STRIDED) offb[i] = strided_lane_offset<T::BN>(wave * T::BB + i, lane, cols_valid, ldw);
        else offb[i] = lane_offset<T>(wave * T::BB + i, lane, cols_valid, ldw);
    }
    // load l of the wavefront's LOADS loads of a k-tile: first the AB blocks of A, then the BB blocks of W (k-tiles are
    // issued in ascending order; load 0 of a k-tile comes first)
    const uint32_t lds_a = lds0 + wave * T::AB * 1024, lds_b = lds0 + T::A_STAGE + wave * T::BB * 1024;
    auto aim = [&](uint32_t stage, auto l_c) __attribute__((always_inline)) {
        constexpr int l = decltype(l_c)::value;
        if constexpr (l < T::AB) set_lds_target<l * 1024>(lds_a + stage);
        else set_lds_target<(l - T::AB) * 1024>(lds_b + stage);
    };
    auto load = [&](int kt, auto l_c) __attribute__((always_inline)) {
        constexpr int l = decltype(l_c)::value;
        if constexpr (l == 0) pa.seek(kt);
        if constexpr (l < T::AB) load_to_lds_16(pa.at(kt), pa.off[l]);
        else if constexpr (LayB::STRIDED) load_to_lds_16(wt + kt * (ldw * T::BK), offb[l - T::AB]);
        else load_to_lds_16(wt + (int64_t)kt * T::BK, offb[l - T::AB]);
    };

    // LDS -> fragment addresses: lane reads row (lane%16) of a 16-row block, k-slot 4*half + lane/16,
    // un-swizzled by the row's swizzle, which only depends on the lane
    const int frow = lane & 15, fh = lane >> 4, fs = (frow >> 1) & 7;
    const int a_base = (wm * T::WTM + frow) * T::ROWB;
    const int b_base = T::A_STAGE + (wn * T::WTN + frow) * T::ROWB;
    // ... of KStrided operands: the lane's row among 32 and its place in the row, and the swizzle of it in bytes
    const int trow = 8 * fh + (frow >> 2);
    const uint32_t t_low = ((frow & 3) >> 1) * 16 + (frow & 1) * 8;
    uint32_t ta_lane = 0, ta_swz = 0, tb_lane = 0, tb_swz = 0;
    if constexpr (LayA::STRIDED) {
        ta_lane = lds0 + trow * T::BM * 2 + t_low;
        ta_swz = strided_swizzle<T::BM>(trow) * 16;
    }
    if constexpr (LayB::STRIDED) {
        tb_lane = lds0 + T::A_STAGE + trow * T::BN * 2 + t_low;
        tb_swz = strided_swizzle<T::BN>(trow) * 16;
    }
    bf16x8_t fa[2][T::FM], fb[2][T::FN];
    auto read_a = [&](uint32_t stage, auto half_c, auto i_c) __attribute__((always_inline)) {
        constexpr int half = decltype(half_c)::value, i = decltype(i_c)::value;
        if constexpr (LayA::STRIDED) {
            fa[half][i] = strided_fragment<T::BM>(stage + half * 32 * T::BM * 2 + ta_lane + (((wm * T::WTM + i * 16) * 2) ^ ta_swz));
        } else {
            const int slot = ((4 * half + fh) ^ fs) << 4;
            const unsigned char *base = smem + stage + slot;
            fa[half][i] = *reinterpret_cast<const bf16x8_t *>(base + a_base + i * 16 * T::ROWB);
        }
    };
    auto read_b = [&](uint32_t stage, auto half_c, auto j_c) __attribute__((always_inline)) {
        constexpr int half = decltype(half_c)::value, j = decltype(j_c)::value;
        if constexpr (LayB::STRIDED) {
            fb[half][j] = strided_fragment<T::BN>(stage + half * 32 * T::BN * 2 + tb_lane + (((wn * T::WTN + j * 16) * 2) ^ tb_swz));
        } else {
            const int slot = ((4 * half + fh) ^ fs) << 4;
            const unsigned char *base = smem + stage + slot;
            fb[half][j] = *reinterpret_cast<const bf16x8_t *>(base + b_base + j * 16 * T::ROWB);
        }
    };
    // fragment q of the FM + FN fragments of a half: the order of their first use (row block 0, every column block,
    // the other row blocks)
    auto read_frag = [&](uint32_t stage, auto half_c, auto q_c) __attribute__((always_inline)) {
        constexpr int q = decltype(q_c)::value;
        if constexpr (q == 0) read_a(stage, half_c, std::integral_constant<int, 0>{});
        else if constexpr (q <= T::FN) read_b(stage, half_c, std::integral_constant<int, q - 1>{});
        else read_a(stage, half_c, std::integral_constant<int, q - T::FN>{});
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};

    // Past the last k-tile the loads go on, on the last k-tile again and into stages that are not read any more: every
    // turn is then the same code, which is what keeps the accumulators where they are (with a turn of its own for the
    // end of a tile the compiler copies all 256 of them between the two).
    const int KT = scalar(K) / T::BK;
    // ---- prologue: the loads of the first D k-tiles, except those that turn 0 issues itself
    static_for<D>([&](auto d) __attribute__((always_inline)) {
        static_for<T::LOADS>([&](auto l) __attribute__((always_inline)) {
            if constexpr (d.value < D - 1 || l.value < T::LOADS - T::WRAPPED) {
                aim(d.value * T::STAGE, l);
                asm volatile("s_nop 0" ::: "memory");
                load(min(d.value, KT - 1), l);
            }
        });
    });
    wait_vmem<(D - 1) * T::LOADS - T::WRAPPED>();
    wg_barrier();                          // k-tile 0 has landed for everyone
    after_first_wait();
    static_for<T::NR>([&](auto q) __attribute__((always_inline)) { read_frag(0, first, q); });

    if constexpr (T::at(T::TT - T::LS, T::LSTEP, T::LOADS)) aim((D - 1) * T::STAGE, std::integral_constant<int, (T::TT - T::LS) / T::LSTEP>{});
    uint32_t st_prev = (D - 1) * T::STAGE, st_cur = 0;         // byte offsets in the ring of the stages of k-tiles k - 1 and k
#pragma clang loop unroll(disable)
    for (int k = 0; k < KT; ++k) {
        const uint32_t st_next = st_cur == (D - 1) * T::STAGE ? 0 : st_cur + T::STAGE;
        const int kt = min(k + D, KT - 1), kt_wrapped = min(k + D - 1, KT - 1);
        static_for<T::TT>([&](auto p_c) __attribute__((always_inline)) {
            constexpr int p = decltype(p_c)::value;
            constexpr int half = p / T::NM, w = p % T::NM, i = w / T::FN;
            constexpr int j = i % 2 ? T::FN - 1 - w % T::FN : w % T::FN;       // back and forth: one operand stays from MFMA to MFMA
            mfma_16x16x32(acc[j][i], fb[half][j], fa[half][i]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (T::at(p - T::R1, T::RSTEP, T::NR)) read_frag(st_cur, second, std::integral_constant<int, (p - T::R1) / T::RSTEP>{});
            if constexpr (p == T::FREE) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if constexpr (T::FREE == T::LAND) wait_vmem<T::younger_at_land()>();
                wg_barrier();
            }
            if constexpr (p == T::LAND && T::FREE != T::LAND) {
                wait_vmem<T::younger_at_land()>();
                wg_barrier();
            }
            // a load, then the target of the next slot's
            if constexpr (T::at(p + T::TT - T::LS, T::LSTEP, T::LOADS)) load(kt_wrapped, std::integral_constant<int, (p + T::TT - T::LS) / T::LSTEP>{});
            if constexpr (T::at(p - T::LS, T::LSTEP, T::LOADS)) load(kt, std::integral_constant<int, (p - T::LS) / T::LSTEP>{});
            constexpr int n = (p + 1) % T::TT;
            if constexpr (T::at(n + T::TT - T::LS, T::LSTEP, T::LOADS))
                aim(p + 1 < T::TT ? st_prev : st_cur, std::integral_constant<int, (n + T::TT - T::LS) / T::LSTEP>{});
            if constexpr (T::at(n - T::LS, T::LSTEP, T::LOADS)) aim(st_cur, std::integral_constant<int, (n - T::LS) / T::LSTEP>{});
            // (in a tile's last turn these read a stage that is not used again)
            if constexpr (T::at(p - T::R0, T::RSTEP, T::NR)) read_frag(st_next, first, std::integral_constant<int, (p - T::R0) / T::RSTEP>{});
            if constexpr (T::at(p + T::TT - T::R0, T::RSTEP, T::NR)) read_frag(st_cur, first, std::integral_constant<int, (p + T::TT - T::R0) / T::RSTEP>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        st_prev = st_cur;
        st_cur = st_next;
    }
    // accumulators may be read after the last MFMA's 16 passes
    asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    }
}

template <class T, class Hook = NoHook>
static __device__ __forceinline__ void tile_accumulate(TileAcc<T> &ta, const uint16_t *__restrict__ a_tile, int rows_valid,
                                                       const uint16_t *__restrict__ wt_tile, int cols_valid,
                                                       int64_t lda, int64_t ldw, int K, unsigned char *smem,
                                                       Hook after_first_wait = Hook())
{
    PlainA<T> pa(a_tile, rows_valid, lda, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), threadIdx.x & 63);
    tile_accumulate_from<T, Hook, PlainA<T>>(ta, pa, wt_tile, cols_valid, ldw, K, smem, after_first_wait);
}

// Rounds the accumulators to bf16 (nearest even) and stores the valid part of the tile.
// acc[j][i][v] is C[m][n] with m = wm*WTM + 16 i + lane%16, n = wn*WTN + 16 j + 4 (lane/16) + v. The lanes of odd rows
// of 16 exchange their half of column block j for their neighbours' half of block j + 1 (v_permlane16_swap), after
// which a lane holds 8 consecutive columns: a store instruction writes 16 bytes per lane, 64 bytes in each of 16 rows,
// and the two instructions of 64 columns whole lines. (8-byte stores without the exchange: twice the requests, and
// with the conversion done in integer arithmetic 6700 cycles more per 256x256 tile; M 65536, K 4096, N 14336: 5281 ->
// 5124 us.) THROUGH: written through the caches (system scope), for output that a copy engine reads while the kernel
// runs on. N and with it cols_valid are multiples of 8.
template <class T, bool THROUGH = false>
static __device__ __forceinline__ void tile_store(const TileAcc<T> &ta, uint16_t *__restrict__ c_tile, int rows_valid,
                                                  int cols_valid, int64_t ldc)
{
    const f32x4_t (&acc)[T::FN][T::FM] = ta.acc;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / T::WGN, wn = wave % T::WGN;
    const int frow = lane & 15, fh = lane >> 4;
    const int n0 = wn * T::WTN + (fh & 1) * 16 + (fh >> 1) * 8;
#pragma unroll
    for (int i = 0; i < T::FM; ++i) {
        const int m = wm * T::WTM + i * 16 + frow;
        uint16_t *crow = c_tile + (int64_t)m * ldc;
#pragma unroll
        for (int j = 0; j < T::FN; j += 2) {
            const auto lo = __builtin_amdgcn_permlane16_swap(pack2_bf16_rne(acc[j][i][0], acc[j][i][1]),
                                                             pack2_bf16_rne(acc[j + 1][i][0], acc[j + 1][i][1]), false, false);
            const auto hi = __builtin_amdgcn_permlane16_swap(pack2_bf16_rne(acc[j][i][2], acc[j][i][3]),
                                                             pack2_bf16_rne(acc[j + 1][i][2], acc[j + 1][i][3]), false, false);
            const u32x4_t v = {lo[0], hi[0], lo[1], hi[1]};
            const int n = n0 + j * 16;
            if (m < rows_valid && n < cols_valid) {
                if constexpr (THROUGH) store_through_16(crow + n, v);
                else *reinterpret_cast<u32x4_t *>(crow + n) = v;
            }
        }
    }
}

template <class T>
static __device__ __forceinline__ void compute_tile(const uint16_t *__restrict__ a_tile, int rows_valid,
                                                    const uint16_t *__restrict__ wt_tile, int cols_valid,
                                                    uint16_t *__restrict__ c_tile, int64_t lda, int64_t ldw,
                                                    int64_t ldc, int K, unsigned char *smem)
{
    TileAcc<T> ta;
    tile_zero(ta);
    tile_accumulate<T>(ta, a_tile, rows_valid, wt_tile, cols_valid, lda, ldw, K, smem);
    tile_store<T>(ta, c_tile, rows_valid, cols_valid, ldc);
}

// Workgroups are dispatched round-robin over the 8 XCDs (each with its own L2). The tiles are cut
// into 8 runs of consecutive logical ids, one per XCD, and the tile grid is walked in groups of
// group_m row tiles, so that one XCD works on few A row tiles and W column tiles at a time. A launch
// with more tiles than the machine holds workgroups is started with that many workgroups only, and a
// workgroup takes every stride-th tile of its XCD's run: what is in flight on an XCD is the same run of
// ids that one workgroup per tile would give, without a workgroup start per tile.
struct XcdRun { int start, count, first, stride; };
static __device__ __forceinline__ XcdRun xcd_run(int pid, int grid, int total)
{
    const int q = total >> 3, r = total & 7;
    const int xcd = pid & 7;
    return {xcd < r ? xcd * (q + 1) : r * (q + 1) + (xcd - r) * q, q + (xcd < r ? 1 : 0), pid >> 3, (grid - xcd + 7) >> 3};
}

typedef TileCfg<256, 256, 2, 2, 2> T256x256;
typedef TileCfg<128, 128, 2, 2, 2> T128x128;       // two workgroups per CU: for launches that fill the machine
typedef TileCfg<128, 128, 2, 2, 4> T128x128D;      // deep ring, one workgroup per CU: for launches that do not
typedef TileCfg<256, 128, 2, 2, 3> T256x128;
typedef TileCfg<128, 256, 2, 2, 3> T128x256;
typedef TileCfg<64, 256, 1, 4, 3> T64x256;
typedef TileCfg<32, 256, 1, 4, 4> T32x256;
typedef TileCfg<128, 192, 2, 2, 3> T128x192;       // column counts that are multiples of 192 but not of 256
typedef TileCfg<256, 192, 2, 2, 2> T256x192;
// For launches that leave CUs idle with every larger tile. A CU draws 45-52 bytes a cycle from beyond its L2, about 32 when
// all of them do, whatever the tile, so a k-tile's time is its bytes: 24 KiB in 0.24-0.27 us here, 32 KiB in 0.31-0.40 with
// 128x128, and a short launch gains by spreading over more CUs. Six stages keep 120 KiB of loads in flight. M 1024, K 4096,
// N 768 30.6 -> 24.6 us.
typedef TileCfg<64, 128, 2, 2, 6> T64x128;
typedef TileCfg<64, 64, 2, 2, 8> T64x64;           // parts (is_part), rings of four and six pairs of stages
typedef TileCfg<32, 64, 2, 2, 12> T32x64;

// every tile shape, for the dispatch switches below
#define FICCO_FOR_EACH_TILE(X) \
    X(TILE_256x256, T256x256) X(TILE_128x128, T128x128) X(TILE_256x128, T256x128) X(TILE_128x256, T128x256) \
    X(TILE_64x256, T64x256) X(TILE_32x256, T32x256) X(TILE_128x128D, T128x128D) X(TILE_128x192, T128x192) \
    X(TILE_256x192, T256x192) X(TILE_64x128, T64x128) \
    X(TILE_64x64, T64x64) X(TILE_32x64, T32x64)

}  // namespace ficco

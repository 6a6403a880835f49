// bf16 MFMA GEMM kernels for gfx950 (CDNA4): C[rows, N] = A[rows, K] * W[K, N], fp32 accumulate,
// one round-to-nearest-even to bf16 at the end.
//
// This is the "chunk GEMM" of the overlap path (paper Sec. II-B for the operation, Sec. V-A for
// launching it per landed piece or per step). Two entry kernels share one tile routine:
//   * gemm_blocks_kernel   - one launch over a list of equal-height row blocks (a monolithic GEMM,
//                            one landed piece, or the G pieces of a fused step read in place);
//   * gemm_resident_kernel - one launch for the whole run; workgroups draw tiles from a ticket
//                            counter in arrival order and wait until the tile's piece is ready.
//
// Data flow per workgroup tile (BM x BN, 256 threads = 4 wavefronts of 64):
//   global --global_load_lds_dwordx4--> LDS (a ring of stages of BK = 64, XOR-swizzled 16 B slots)
//   LDS --ds_read_b128--> 8-element bf16 fragments --> v_mfma_f32_16x16x32_bf16 --> fp32 accumulators
// The weight is read from a packed copy Wt[N, K] (k contiguous), so A and Wt fragments use the
// same access pattern. Every output element is accumulated over k ascending by the same
// instruction, whatever the tile shape or row block, which makes results bit-identical across
// schedules.
#include "ficco_internal.h"
#include "ficco_gate.h"
#include "ficco_tile.h"
#include <stdlib.h>
#include <algorithm>

namespace ficco {

template <class T>
__global__ __launch_bounds__(T::THREADS) void gemm_blocks_kernel(GemmLaunch a)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    if (a.n_wait > 0) {
        __shared__ int s_go;
        if (threadIdx.x < 64) {
            const int ok = wait_ready_all(a.gate, a.n_wait, pace_of(gridDim.x, gridDim.x), [&](int i) { return a.wait_chunks[i]; });
            if (threadIdx.x == 0) s_go = ok;
        }
        __syncthreads();                   // also orders the tile's loads after the flag reads
        if (!s_go) return;
    }
    const int tiles_n = (a.N + T::BN - 1) / T::BN;
    const int rt_per_block = (a.rows_per_block + T::BM - 1) / T::BM;
    const int tiles_m = a.n_blocks * rt_per_block;
    const int total = tiles_m * tiles_n;
    const XcdRun run = xcd_run(blockIdx.x, gridDim.x, total);
    const int per_group = a.group_m * tiles_n;
    for (int t = run.first; t < run.count; t += run.stride) {
        const int lid = run.start + t;
        const int group = lid / per_group;
        const int first_m = group * a.group_m;
        const int gsz = min(tiles_m - first_m, a.group_m);
        const int tm = first_m + (lid % per_group) % gsz;
        const int tn = (lid % per_group) / gsz;

        const int blk = tm / rt_per_block, rt = tm % rt_per_block;
        const int brow0 = a.block_row0 ? a.block_row0[blk] : a.row0;
        const int64_t row0 = (int64_t)brow0 + (int64_t)rt * T::BM;
        const int rows_valid = min(T::BM, a.rows_per_block - rt * T::BM);
        const int col0 = tn * T::BN;
        const int cols_valid = min(T::BN, a.N - col0);
        compute_tile<T>(a.A + row0 * a.lda, rows_valid, a.Wt + (int64_t)col0 * a.K, cols_valid,
                        a.C + row0 * a.ldc + col0, a.lda, a.K, a.ldc, a.K, smem);
        __syncthreads();                   // everyone is done with the ring before the next tile refills it
    }
    wait_vmem<0>();                        // no load may arrive in LDS that is not this workgroup's any more
}

// Tile order of the resident kernels. Row tiles are numbered in arrival order (R = arrival position x
// row tiles per piece + row tile in the piece) and dealt round-robin to kTicketLists lists, one per
// XCD, each with its own ticket counter: a workgroup first serves the list of the XCD it presumably
// runs on (workgroups are dispatched round-robin over the XCDs), so that the tiles sharing an L2 at
// any time are few row tiles times a run of column tiles, and then helps the other lists. Inside a
// list tiles go in groups of a few row tiles, row tile fastest: as many as one step delivers to the
// list (so that no workgroup draws a tile of the next step while tiles of this one are left), 1 to 8.
// When a step delivers few row tiles and there are many column tiles, one row tile times all columns
// per XCD would stream the whole weight through every L2 once per round; the row-piece kernel then
// splits the lists by column block as well (ResidentLaunch::col_lists), so that an XCD works on
// several row tiles of the step times a run of columns, as a launch over the step's pieces would.
//
// TileWalk hands a workgroup its next (list, tile) pair. The first `rounds` tiles of its home list are the workgroup's
// by its rank among the workgroups that start there (no memory access), and short launches have all their tiles that way
// (hand_out); later tiles are drawn from the list's counter. Before it turns to the other lists it reads their counters once, all
// loads in flight together: on a list that is already used up it only leaves its one past-the-end draw (an atomic
// whose result nobody waits for), and a list that the ranks of its own workgroups cover completely is never drawn from
// at all. Counter traffic is what a launch pays at its end, since a draw goes to memory shared by all XCDs.
struct TileWalk {
    int turn;        // lists visited so far; the current list is (home + turn) % kTicketLists
    int taken;       // tiles of the home list taken by rank so far
    int looked;      // the other lists' counters have been read
    int spent;       // bit k: list (home + k) % kTicketLists was already used up at that look
    int x, t;        // the result: list and tile in the list, x < 0 when there is nothing left
    int have_drawn;  // `drawn` holds a counter value drawn ahead of time (kept here and not in a register across the k
    uint32_t drawn;  // loop, which leaves none: the compiler would spill it to memory)
};

// Issues, ahead of time, the draw that the next tile_walk_next() call would start with (if it would
// start with one) and returns 1 with the raw counter value in `drawn`; the caller puts this before
// work whose duration then hides the draw's round trip. Returns 0 when the next step is not a plain draw.
template <class TotalFn>
static __device__ __forceinline__ int tile_walk_predraw(const TileWalk &w, uint32_t *ticket, int grid, HandOut out, TotalFn total_of,
                                                        uint32_t &drawn)
{
    const int rounds = out.rounds;
    if (out.by_rank || w.turn >= kTicketLists || (w.turn == 0 && w.taken < rounds)) return 0;
    const int y = (blockIdx.x + w.turn) % kTicketLists;
    if (total_of(y) <= rounds * resident_list_homes(grid, y)) return 0;
    if (w.turn > 0 && (!w.looked || ((w.spent >> w.turn) & 1))) return 0;
    drawn = __hip_atomic_fetch_add(ticket + y * kFlagStrideWords, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return 1;
}

template <class TotalFn>
static __device__ __forceinline__ void tile_walk_next(TileWalk &w, uint32_t *ticket, const uint32_t *base, int grid, HandOut out,
                                                      TotalFn total_of)
{
    const int home = blockIdx.x % kTicketLists, rank = blockIdx.x / kTicketLists, rounds = out.rounds;
    w.x = -1;
    if (__builtin_expect(out.by_rank, 0)) {
        if (w.taken < rounds && !tile_by_rank(home, rank, w.taken, grid, rounds, total_of, w.x, w.t)) w.taken = rounds;
        ++w.taken;
        return;
    }
    while (w.turn < kTicketLists) {
        const int y = (home + w.turn) % kTicketLists;
        const int total = total_of(y), homes = resident_list_homes(grid, y);
        uint32_t *ctr = ticket + y * kFlagStrideWords;
        if (w.turn == 0 && w.taken < rounds) {
            const int cand = rank + w.taken * homes;
            ++w.taken;
            if (cand < total) { w.x = y; w.t = cand; return; }
            w.taken = rounds;                      // and none further on
        }
        if (total <= rounds * homes) {
            // the ranks of the workgroups that start on this list cover it: nobody draws from its counter
            ++w.turn;
            continue;
        }
        if (w.turn > 0 && !w.looked) {
            uint32_t seen[kTicketLists];
#pragma unroll
            for (int k = 1; k < kTicketLists; ++k)
                seen[k] = __hip_atomic_load(ticket + ((home + k) % kTicketLists) * kFlagStrideWords, __ATOMIC_RELAXED,
                                            __HIP_MEMORY_SCOPE_AGENT);
            int spent = 0;
#pragma unroll
            for (int k = 1; k < kTicketLists; ++k) {
                const int yk = (home + k) % kTicketLists;
                const int by_rank = rounds * resident_list_homes(grid, yk), total_k = total_of(yk);
                if (total_k > by_rank && (int)(seen[k] - base[yk]) + by_rank >= total_k) spent |= 1 << k;
            }
            w.spent = spent;
            w.looked = 1;
        }
        if (w.turn > 0 && ((w.spent >> w.turn) & 1)) {
            (void)__hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // result unused: no wait
            ++w.turn;
            continue;
        }
        const uint32_t raw = w.have_drawn ? w.drawn : __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        w.have_drawn = 0;
        const int cand = (int)(raw - base[y]) + rounds * homes;
        if (cand < total) { w.x = y; w.t = cand; return; }
        ++w.turn;                                  // that was this workgroup's one draw past the end of list y
    }
}

// The lists of a resident launch as a grid of row classes x column blocks (see resident_list_tiles):
// which tiles list x holds and where tile t of it lies. Inside a list tiles go in groups of `group`
// row tiles, row tile fastest.
struct ListGrid {
    int row_tiles, tiles_n, group;
    int cl_shift;                // log2 of the number of column blocks (1, 2, 4 or 8 of them): shifts, not divisions
    __device__ __forceinline__ ListGrid(int row_tiles_, int tiles_n_, int col_lists, int group_)
        : row_tiles(row_tiles_), tiles_n(tiles_n_), group(group_), cl_shift(31 - __clz(col_lists)) {}
    __device__ __forceinline__ int class_shift() const { return 3 - cl_shift; }              // kTicketLists = 8 lists
    __device__ __forceinline__ int row_class(int x) const { return x & ((1 << class_shift()) - 1); }
    __device__ __forceinline__ int col_block(int x) const { return x >> class_shift(); }
    __device__ __forceinline__ int rows(int x) const
    {
        const int rc = row_class(x);
        return row_tiles > rc ? (row_tiles - rc + (1 << class_shift()) - 1) >> class_shift() : 0;
    }
    __device__ __forceinline__ int col_begin(int x) const { return (col_block(x) * tiles_n) >> cl_shift; }
    __device__ __forceinline__ int cols(int x) const { return (((col_block(x) + 1) * tiles_n) >> cl_shift) - col_begin(x); }
    __device__ __forceinline__ int total(int x) const { return rows(x) * cols(x); }
    // tile t of list x: R = its row tile in the arrival-ordered sequence, tn = its column tile
    __device__ __forceinline__ void position(int x, int t, int &R, int &tn) const
    {
        const int my_rows = rows(x), my_cols = cols(x);
        const int per_group = group * my_cols;
        const int g = t / per_group, first = g * group;
        const int gsz = min(my_rows - first, group);
        R = ((first + (t % per_group) % gsz) << class_shift()) + row_class(x);
        tn = col_begin(x) + (t % per_group) / gsz;
    }
};
static_assert(kTicketLists == 8, "ListGrid shifts assume 8 lists");

// A workgroup of a resident kernel has read everything it will read of A when it gets here (the data went
// through the MFMAs before its last tile was stored), so the last one out may let the next run's transfers
// into A start.
__device__ __forceinline__ void leave_run(const RunExit &e)
{
    if (e.release_value && threadIdx.x == 0) {
        const uint32_t before = __hip_atomic_fetch_add(e.count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before + 1u == e.target)
            __hip_atomic_store(e.release_value, (int64_t)0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
    }
}

// STREAM_OUT: the GEMM -> reduce-scatter form (r.done_count set), a separate instantiation so that its
// epilogue and bookkeeping cost the all-gather form no registers.
template <class T, bool STREAM_OUT>
__global__ __launch_bounds__(T::THREADS) void gemm_resident_kernel(ResidentLaunch r)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    __shared__ TileWalk s_walk;
    __shared__ int s_ok, s_chunk;
    const GemmLaunch &a = r.g;
    const int tiles_n = (a.N + T::BN - 1) / T::BN;
    const int rt_per_chunk = (a.rows_per_block + T::BM - 1) / T::BM;
    const int row_tiles = r.n_chunks * rt_per_chunk;
    const ListGrid lists(row_tiles, tiles_n, r.col_lists, r.group);
    auto total_of = [&](int x) { return lists.total(x); };

    if (threadIdx.x == 0) s_walk = TileWalk{0, 0, 0, 0, -1, 0, 0, 0};
    // Output streaming: a copy engine reads a piece of C while the kernel runs on, so
    // the tiles are written through the caches, and a tile is counted for its piece once every thread's
    // stores have been performed; whoever completes a piece lets its copy go. Ordering is by hand
    // (stores, their completion, barrier, counter, signal): a release fence would write back the whole
    // L2 once per tile. So that nobody waits for stores, a tile is counted under the next tile's
    // first k-step, or after the loop if it was the workgroup's last.
    int stored_chunk = -1;                 // thread 0: piece of the tile stored last and not yet counted
    auto count_stored = [&]() {
        if (STREAM_OUT && threadIdx.x == 0 && stored_chunk >= 0) {
            const uint32_t before = __hip_atomic_fetch_add(r.done_count + stored_chunk, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if ((before + 1u) % (uint32_t)r.tiles_per_chunk == 0u)
                __hip_atomic_store(reinterpret_cast<int64_t *>(r.done_sig[stored_chunk]), (int64_t)0, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_SYSTEM);
            stored_chunk = -1;
        }
    };
    for (;;) {
        if (threadIdx.x == 0) {
            TileWalk w = s_walk;
            tile_walk_next(w, r.ticket, r.ticket_base, r.grid, r.out, total_of);
            int ok = 1;
            if (w.x >= 0) {
                int R, tn;
                lists.position(w.x, w.t, R, tn);
                const int chunk = r.arrival[R / rt_per_chunk];
                if (chunk < r.local_chunk_begin || chunk >= r.local_chunk_end) ok = wait_ready(gate_argument(offsetof(ResidentLaunch, g.gate)), chunk, pace_of(r.grid, rt_per_chunk * tiles_n));
                s_chunk = chunk;           // the others take it from here instead of the table in memory
            }
            s_walk = w;
            s_ok = ok;
        }
        __syncthreads();                   // also orders the tile's loads after the flag read
        const int x = __builtin_amdgcn_readfirstlane(s_walk.x), t = __builtin_amdgcn_readfirstlane(s_walk.t);
        if (x < 0) break;
        if (s_ok) {
            int R, tn;
            lists.position(x, t, R, tn);
            const int rt = R % rt_per_chunk;
            const int chunk = __builtin_amdgcn_readfirstlane(s_chunk);
            const int64_t row0 = (int64_t)chunk * a.rows_per_block + (int64_t)rt * T::BM;
            const int rows_valid = min(T::BM, a.rows_per_block - rt * T::BM);
            const int col0 = tn * T::BN;
            const int cols_valid = min(T::BN, a.N - col0);
            TileAcc<T> ta;
            tile_zero(ta);
            if constexpr (STREAM_OUT)
                tile_accumulate<T>(ta, a.A + row0 * a.lda, rows_valid, a.Wt + (int64_t)col0 * a.K, cols_valid, a.lda, a.K, a.K, smem,
                                   count_stored);
            else
                tile_accumulate<T>(ta, a.A + row0 * a.lda, rows_valid, a.Wt + (int64_t)col0 * a.K, cols_valid, a.lda, a.K, a.K, smem);
            // the next ticket's round trip runs under the epilogue
            int have_drawn = 0;
            uint32_t drawn = 0;
            if (threadIdx.x == 0) have_drawn = tile_walk_predraw(s_walk, r.ticket, r.grid, r.out, total_of, drawn);
            if constexpr (STREAM_OUT) {
                tile_store<T, true>(ta, a.C + row0 * a.ldc + col0, rows_valid, cols_valid, a.ldc);
                stored_chunk = chunk;
            } else {
                tile_store<T>(ta, a.C + row0 * a.ldc + col0, rows_valid, cols_valid, a.ldc);
            }
            if (threadIdx.x == 0) { s_walk.have_drawn = have_drawn; s_walk.drawn = drawn; }
        }
        __syncthreads();                   // s_walk / s_ok / LDS stages are reused
    }
    wait_vmem<0>();                        // no load may arrive in LDS that is not this workgroup's any more; stores are done
    if constexpr (STREAM_OUT) {
        __syncthreads();
        count_stored();
    }
    leave_run(r.leave);
}

// Column-piece variant of the resident kernel (the 2D communication shape of Sec. V-A, chosen when
// M <= K): step s delivers K-slice s of every shard, and every tile of C can make progress at every
// step. The accumulation order over k is that of the monolithic kernel, so the bits are the same.
template <class T>
__global__ __launch_bounds__(T::THREADS) void gemm_resident2d_kernel(Resident2DLaunch r)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    __shared__ TileWalk s_walk;
    __shared__ int s_ok;
    const GemmLaunch &a = r.g;
    const int tiles_n = (a.N + T::BN - 1) / T::BN;
    const int row_tiles = (r.M + T::BM - 1) / T::BM;
    const ListGrid lists(row_tiles, tiles_n, r.col_lists, r.group);
    auto total_of = [&](int x) { return lists.total(x); };

    if (threadIdx.x == 0) s_walk = TileWalk{0, 0, 0, 0, -1, 0, 0, 0};
    for (;;) {
        if (threadIdx.x == 0) {
            TileWalk w = s_walk;
            tile_walk_next(w, r.ticket, r.ticket_base, r.grid, r.out, total_of);
            s_walk = w;
        }
        __syncthreads();
        const int x = __builtin_amdgcn_readfirstlane(s_walk.x), t = __builtin_amdgcn_readfirstlane(s_walk.t);
        if (x < 0) break;
        int tm, tn;
        lists.position(x, t, tm, tn);
        const int64_t row0 = (int64_t)tm * T::BM;
        const int rows_valid = min(T::BM, r.M - (int)row0);
        const int col0 = tn * T::BN;
        const int cols_valid = min(T::BN, a.N - col0);
        const int j0 = (int)(row0 / r.rows_per_shard), j1 = (int)((row0 + rows_valid - 1) / r.rows_per_shard);
        TileAcc<T> ta;
        tile_zero(ta);
        int ok = 1;
        // The k loop takes runs of slices: it waits for the next slice, then looks (without waiting) how many of
        // the following ones have landed as well, and multiplies the whole run as one k range, so that the load
        // pipeline is only drained where the kernel has to wait anyway. With operands resident the run is all of K.
        for (int sl = 0; sl < r.slices && ok;) {
            int run_end = r.slices;
            if (r.gated) {
                if (threadIdx.x < 64) {
                    const Gate gate = gate_argument(offsetof(Resident2DLaunch, g.gate));
                    const Pace pace = pace_of(r.grid, r.grid / r.shards);
                    const int o = wait_ready_all(gate, j1 - j0 + 1, pace, [&](int i) { return sl * r.shards + j0 + i; });
                    // one look at up to 64 following slices, a lane each
                    const int mine = sl + 1 + (int)threadIdx.x;
                    int landed = o && mine < r.slices;
                    for (int j = j0; j <= j1; ++j) landed = landed && peek_ready(gate, mine * r.shards + j, pace.every > 1, (poll_phase(blockIdx.x, pace.every) + sl) % pace.every == 0);
                    const uint64_t not_landed = ~__ballot(landed);
                    const int run = not_landed ? __builtin_ctzll(not_landed) : 64;
                    if (threadIdx.x == 0) s_ok = o ? sl + 1 + run : 0;      // 0: gave up; else the slice after the run
                }
                __syncthreads();           // also orders the run's loads after the flag reads
                run_end = s_ok;
                ok = run_end != 0;
                __syncthreads();
            }
            if (ok) {
                const int kb = r.k0[sl], ke = r.k0[run_end];              // the run's columns: [kb, ke)
                SlicedA<T> pa(a.A, r.k0, r.M, row0, sl, rows_valid, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), threadIdx.x & 63);
                tile_accumulate_from<T, NoHook, SlicedA<T>>(ta, pa, a.Wt + (int64_t)col0 * a.K + kb, cols_valid, a.K, ke - kb, smem);
                sl = run_end;
            }
        }
        int have_drawn = 0;
        uint32_t drawn = 0;
        if (threadIdx.x == 0) have_drawn = tile_walk_predraw(s_walk, r.ticket, r.grid, r.out, total_of, drawn);
        if (ok) tile_store<T>(ta, a.C + row0 * a.ldc + col0, rows_valid, cols_valid, a.ldc);
        if (threadIdx.x == 0) { s_walk.have_drawn = have_drawn; s_walk.drawn = drawn; }
        __syncthreads();                   // s_walk / s_ok / LDS stages are reused
    }
    wait_vmem<0>();                        // no load may arrive in LDS that is not this workgroup's any more
    leave_run(r.leave);
}

// Expert-parallel variant of the resident kernel (all-to-all token dispatch before the expert layers,
// Sec. II-A; unequal amounts per pair of GPUs, Sec. III-C): the rows of A are ragged segments, one per
// expert, each multiplied by that expert's weight. Row tiles never cross a segment; the host lists
// them in the order they become ready together with the pieces that cover them.
template <class T>
__global__ __launch_bounds__(T::THREADS) void gemm_grouped_kernel(GroupedLaunch r)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    __shared__ TileWalk s_walk;
    __shared__ int s_ok;
    const GemmLaunch &a = r.g;
    const int tiles_n = (a.N + T::BN - 1) / T::BN;
    const ListGrid lists(r.n_row_tiles, tiles_n, r.col_lists, r.group);
    auto total_of = [&](int x) { return lists.total(x); };

    if (threadIdx.x == 0) s_walk = TileWalk{0, 0, 0, 0, -1, 0, 0, 0};
    for (;;) {
        if (threadIdx.x < 64) {
            TileWalk w{};
            if (threadIdx.x == 0) {
                w = s_walk;
                tile_walk_next(w, r.ticket, r.ticket_base, r.grid, r.out, total_of);
                s_walk = w;
            }
            const int wx = __builtin_amdgcn_readfirstlane(w.x), wt = __builtin_amdgcn_readfirstlane(w.t);
            int ok = 1;
            if (wx >= 0 && r.gated) {
                int R, tn;
                lists.position(wx, wt, R, tn);
                const int32_t *rt = r.row_tiles + (size_t)R * kRowTileWords;
                const int first = rt[3];
                ok = wait_ready_all(gate_argument(offsetof(GroupedLaunch, g.gate)), rt[4] - first + 1, pace_of(r.grid, tiles_n), [&](int i) { return first + i; });
            }
            if (threadIdx.x == 0) s_ok = ok;
        }
        __syncthreads();                   // also orders the tile's loads after the flag reads
        const int x = __builtin_amdgcn_readfirstlane(s_walk.x), t = __builtin_amdgcn_readfirstlane(s_walk.t);
        if (x < 0) break;
        if (s_ok) {
            int R, tn;
            lists.position(x, t, R, tn);
            const int32_t *rt = r.row_tiles + (size_t)R * kRowTileWords;
            const int64_t row0 = rt[0];
            const int rows_valid = rt[1];
            const int64_t expert = rt[2];
            const int col0 = tn * T::BN;
            const int cols_valid = min(T::BN, a.N - col0);
            TileAcc<T> ta;
            tile_zero(ta);
            tile_accumulate<T>(ta, a.A + row0 * a.lda, rows_valid, a.Wt + (expert * a.N + col0) * (int64_t)a.K, cols_valid,
                               a.lda, a.K, a.K, smem);
            int have_drawn = 0;
            uint32_t drawn = 0;
            if (threadIdx.x == 0) have_drawn = tile_walk_predraw(s_walk, r.ticket, r.grid, r.out, total_of, drawn);
            tile_store<T>(ta, a.C + row0 * a.ldc + col0, rows_valid, cols_valid, a.ldc);
            if (threadIdx.x == 0) { s_walk.have_drawn = have_drawn; s_walk.drawn = drawn; }
        }
        __syncthreads();                   // s_walk / s_ok / LDS stages are reused
    }
    wait_vmem<0>();                        // no load may arrive in LDS that is not this workgroup's any more
}

__global__ __launch_bounds__(64) void wait_ready_kernel(Gate gate, const int32_t *chunks, int n)
{
    (void)wait_ready_all(gate, n, Pace{1, 1}, [&](int i) { return chunks[i]; });
}

// Nothing is published through the signal: what it orders is that the kernels before this one on the
// stream have finished reading A, which stream order has settled when this kernel starts. A relaxed store
// therefore does, and spares the cache write-back a release at system scope would add.
__global__ __launch_bounds__(64) void release_signal_kernel(int64_t *value)
{
    if (threadIdx.x == 0) __hip_atomic_store(value, (int64_t)0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}

// W[K,N] -> Wt[N,K], one wavefront per 64x64 tile, for a 16-byte aligned W, K % 64 == 0 and N % 8 == 0. A lane turns an
// 8x8 block in its registers (eight 16-byte loads, 32 byte permutes, eight 16-byte stores); lane l has k group l % 8 and
// column group l / 8, so that a load instruction reads, and a store instruction writes, whole 128-byte lines.
// Streaming work, bound by memory. The first workgroup also clears `clear_words` words at `clear` for the caller.
__global__ __launch_bounds__(256) void pack_weight_kernel(const uint16_t *__restrict__ W, uint16_t *__restrict__ Wt,
                                                          int64_t K, int64_t N, uint32_t *clear, int clear_words)
{
    if (blockIdx.x == 0 && blockIdx.y == 0 && (int)threadIdx.x < clear_words) clear[threadIdx.x] = 0u;
    const int lane = threadIdx.x & 63;
    const int64_t k0 = ((int64_t)blockIdx.y * 4 + (threadIdx.x >> 6)) * 64 + (lane & 7) * 8, n0 = (int64_t)blockIdx.x * 64 + (lane >> 3) * 8;
    if (k0 >= K || n0 >= N) return;
    u32x4_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = *reinterpret_cast<const u32x4_t *>(W + (k0 + i) * N + n0);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        u32x4_t even, odd;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            even[i] = __builtin_amdgcn_perm(r[2 * i + 1][c], r[2 * i][c], 0x05040100u);
            odd[i] = __builtin_amdgcn_perm(r[2 * i + 1][c], r[2 * i][c], 0x07060302u);
        }
        *reinterpret_cast<u32x4_t *>(Wt + (n0 + 2 * c) * K + k0) = even;
        *reinterpret_cast<u32x4_t *>(Wt + (n0 + 2 * c + 1) * K + k0) = odd;
    }
}

// The same for any W, 2 bytes at a time through a 64x64 LDS tile (padded), 256 threads.
__global__ __launch_bounds__(256) void pack_weight_unaligned_kernel(const uint16_t *__restrict__ W, uint16_t *__restrict__ Wt,
                                                                    int64_t K, int64_t N, uint32_t *clear, int clear_words)
{
    if (blockIdx.x == 0 && blockIdx.y == 0 && (int)threadIdx.x < clear_words) clear[threadIdx.x] = 0u;
    __shared__ uint16_t t[64][66];
    const int64_t k0 = (int64_t)blockIdx.y * 64, n0 = (int64_t)blockIdx.x * 64;
    for (int e = threadIdx.x; e < 64 * 64; e += 256) {
        int kk = e >> 6, nn = e & 63;
        if (k0 + kk < K && n0 + nn < N) t[kk][nn] = W[(k0 + kk) * N + n0 + nn];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 64 * 64; e += 256) {
        int nn = e >> 6, kk = e & 63;
        if (k0 + kk < K && n0 + nn < N) Wt[(n0 + nn) * K + k0 + kk] = t[kk][nn];
    }
}

// Sender-side re-layout of column pieces out of a row-major matrix (see SliceLaunch). 16-byte vectors, a row
// of a piece is width/8 of them; the workgroup's threads stride over (row, vector) pairs of its block.
__global__ __launch_bounds__(256) void slice_source_kernel(SliceLaunch a)
{
    // blocks in arrival order, a bounded number of workgroups striding over them: the pieces of the first step
    // are finished - and their transfers released - first instead of every piece at the end
    const int total_blocks = a.n_pieces * a.blocks_per_piece;
    for (int blk = blockIdx.x; blk < total_blocks; blk += gridDim.x) {
        const int q = blk / a.blocks_per_piece, b = blk % a.blocks_per_piece;
        const int piece = a.arrival[q];
        const int sl = piece / a.shards, j = piece % a.shards;
        const int kb = a.k0[sl], kw = a.k0[sl + 1] - kb;
        const int r0 = b * a.rows_per_block, r1 = min(a.rows_per_shard, r0 + a.rows_per_block);
        const int vecs = kw / 8;
        const u32x4_t *src = reinterpret_cast<const u32x4_t *>(a.src + ((int64_t)j * a.rows_per_shard + r0) * a.K + kb);
        u32x4_t *dst = reinterpret_cast<u32x4_t *>(a.dst + a.M * kb + ((int64_t)j * a.rows_per_shard + r0) * kw);
        const int64_t src_pitch = a.K / 8;
        const int total = (r1 - r0) * vecs;
        for (int e = threadIdx.x; e < total; e += 4 * 256) {
            u32x4_t v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int ee = e + u * 256;
                if (ee < total) v[u] = __builtin_nontemporal_load(src + (int64_t)(ee / vecs) * src_pitch + ee % vecs);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int ee = e + u * 256;
                // written through the caches: the reader is a copy engine
                if (ee < total) store_through_16(dst + ee, v[u]);
            }
        }
        // every store of the block has been performed (not just issued) before the block is counted
        wait_vmem<0>();
        __syncthreads();
        if (threadIdx.x == 0) {
            const uint32_t before = __hip_atomic_fetch_add(a.done_count + piece, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if ((before + 1u) % (uint32_t)a.blocks_per_piece == 0u)
                __hip_atomic_store(reinterpret_cast<int64_t *>(a.done_sig[piece]), (int64_t)0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
        }
    }
}

hipError_t launch_slice_source(const SliceLaunch &a, hipStream_t s)
{
    if (a.n_pieces <= 0 || a.blocks_per_piece <= 0 || a.rows_per_block <= 0) return hipErrorInvalidValue;
    const int64_t total = (int64_t)a.n_pieces * a.blocks_per_piece;
    if (total > 0x7FFFFFFF) return hipErrorInvalidValue;
    hipLaunchKernelGGL(slice_source_kernel, dim3((unsigned)std::min<int64_t>(total, 1024)), dim3(256), 0, s, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------ host
TileShape tile_shape(int tile)
{
    switch (tile) {
#define X(id, T) case id: return {T::BM, T::BN, T::LDS_BYTES, T::THREADS};
    FICCO_FOR_EACH_TILE(X)
#undef X
    default: return {0, 0, 0, 0};
    }
}

template <class T>
static hipError_t launch_gemm_t(const GemmLaunch &a, hipStream_t s)
{
    const hipError_t limit = raise_lds_limit<&gemm_blocks_kernel<T>>(T::LDS_BYTES);
    if (limit != hipSuccess) return limit;
    const int tiles_n = (a.N + T::BN - 1) / T::BN;
    const int rt = (a.rows_per_block + T::BM - 1) / T::BM;
    const int64_t total = (int64_t)a.n_blocks * rt * tiles_n;
    if (total <= 0 || total > 0x7FFFFFFF || a.lda > kMaxK || a.K > kMaxK) return hipErrorInvalidValue;
    // at most as many workgroups as run at once (a multiple of 8, one share per XCD); the rest of the tiles
    // are taken by the kernel's loop
    int64_t grid = total;
    {
        static int fit_of[64];                       // per device: 0 = not asked yet, -1 = could not be asked
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess) return hipGetLastError();
        int fit = dev < 64 ? fit_of[dev] : 0;
        if (fit == 0) {
            int per_cu = 0, cus = 0;
            if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, gemm_blocks_kernel<T>, T::THREADS, T::LDS_BYTES) == hipSuccess &&
                hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && per_cu * cus >= 8)
                fit = per_cu * cus / 8 * 8;
            else
                fit = -1;
            if (dev < 64) fit_of[dev] = fit;
        }
        if (fit > 0 && total > fit) grid = fit;
    }
    // group height of the tile order: matters when the launch runs for several rounds
    GemmLaunch b = a;
    if (b.group_m != 1 && b.group_m != 2 && b.group_m != 4 && b.group_m != 8) b.group_m = 0;
    if (!b.group_m) b.group_m = 8;
    if (!a.group_m && total > grid) {
        double best = -1;
        for (int g = 1; g <= 8; g *= 2) {
            const double c = tile_order_cost(T::BM, T::BN, tiles_n, (int64_t)a.n_blocks * rt, grid / 8, 1, g,
                                             (int64_t)a.n_blocks * a.rows_per_block * a.K * 2, (int64_t)a.N * a.K * 2);
            if (best < 0 || c < best) { best = c; b.group_m = g; }
        }
    }
    hipLaunchKernelGGL(gemm_blocks_kernel<T>, dim3((unsigned)grid), dim3(T::THREADS), T::LDS_BYTES, s, b);
    return hipGetLastError();
}

template <class T>
static hipError_t launch_resident_t(const ResidentLaunch &r, hipStream_t s)
{
    const hipError_t limit = r.done_count ? raise_lds_limit<&gemm_resident_kernel<T, true>>(T::LDS_BYTES) : raise_lds_limit<&gemm_resident_kernel<T, false>>(T::LDS_BYTES);
    if (limit != hipSuccess) return limit;
    if (r.grid <= 0 || r.g.lda > kMaxK || r.g.K > kMaxK) return hipErrorInvalidValue;
    if (r.done_count)
        hipLaunchKernelGGL((gemm_resident_kernel<T, true>), dim3((unsigned)r.grid), dim3(T::THREADS), T::LDS_BYTES, s, r);
    else
        hipLaunchKernelGGL((gemm_resident_kernel<T, false>), dim3((unsigned)r.grid), dim3(T::THREADS), T::LDS_BYTES, s, r);
    return hipGetLastError();
}

template <class T>
static hipError_t launch_resident2d_t(const Resident2DLaunch &r, hipStream_t s)
{
    const hipError_t limit = raise_lds_limit<&gemm_resident2d_kernel<T>>(T::LDS_BYTES);
    if (limit != hipSuccess) return limit;
    if (r.grid <= 0 || !r.k0 || r.g.K > kMaxK) return hipErrorInvalidValue;
    hipLaunchKernelGGL(gemm_resident2d_kernel<T>, dim3((unsigned)r.grid), dim3(T::THREADS), T::LDS_BYTES, s, r);
    return hipGetLastError();
}

template <class T>
static int resident2d_grid_t(int device)
{
    (void)raise_lds_limit<&gemm_resident2d_kernel<T>>(T::LDS_BYTES);
    int per_cu = 0, cus = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, gemm_resident2d_kernel<T>, T::THREADS, T::LDS_BYTES) != hipSuccess) return 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess) return 0;
    return per_cu * cus;
}

template <class T>
static hipError_t launch_grouped_t(const GroupedLaunch &r, hipStream_t s)
{
    const hipError_t limit = raise_lds_limit<&gemm_grouped_kernel<T>>(T::LDS_BYTES);
    if (limit != hipSuccess) return limit;
    if (r.grid <= 0 || r.n_row_tiles <= 0 || r.g.lda > kMaxK || r.g.K > kMaxK) return hipErrorInvalidValue;
    hipLaunchKernelGGL(gemm_grouped_kernel<T>, dim3((unsigned)r.grid), dim3(T::THREADS), T::LDS_BYTES, s, r);
    return hipGetLastError();
}

template <class T>
static int grouped_grid_t(int device)
{
    (void)raise_lds_limit<&gemm_grouped_kernel<T>>(T::LDS_BYTES);
    int per_cu = 0, cus = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, gemm_grouped_kernel<T>, T::THREADS, T::LDS_BYTES) != hipSuccess) return 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess) return 0;
    return per_cu * cus;
}

template <class T>
static int resident_grid_t(int device)
{
    (void)raise_lds_limit<&gemm_resident_kernel<T, false>>(T::LDS_BYTES);
    int per_cu = 0, cus = 0;
    // (the output-streaming form may need more registers, but every tile shape is limited by LDS first)
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, gemm_resident_kernel<T, false>, T::THREADS, T::LDS_BYTES) != hipSuccess) return 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess) return 0;
    return per_cu * cus;
}


hipError_t launch_gemm(int tile, const GemmLaunch &a, hipStream_t s)
{
    switch (tile) {
#define X(id, T) case id: return launch_gemm_t<T>(a, s);
    FICCO_FOR_EACH_TILE(X)
#undef X
    default: return hipErrorInvalidValue;
    }
}

hipError_t launch_resident(int tile, const ResidentLaunch &r, hipStream_t s)
{
    switch (tile) {
#define X(id, T) case id: return launch_resident_t<T>(r, s);
    FICCO_FOR_EACH_TILE(X)
#undef X
    default: return hipErrorInvalidValue;
    }
}

hipError_t launch_resident2d(int tile, const Resident2DLaunch &r, hipStream_t s)
{
    switch (tile) {
#define X(id, T) case id: return launch_resident2d_t<T>(r, s);
    FICCO_FOR_EACH_TILE(X)
#undef X
    default: return hipErrorInvalidValue;
    }
}

int resident2d_grid_size(int tile, int device)
{
    switch (tile) {
#define X(id, T) case id: return resident2d_grid_t<T>(device);
    FICCO_FOR_EACH_TILE(X)
#undef X
    default: return 0;
    }
}

int resident_grid_size(int tile, int device)
{
    switch (tile) {
#define X(id, T) case id: return resident_grid_t<T>(device);
    FICCO_FOR_EACH_TILE(X)
#undef X
    default: return 0;
    }
}

hipError_t launch_wait_ready(const Gate &gate, const int32_t *chunks, int n, hipStream_t s)
{
    hipLaunchKernelGGL(wait_ready_kernel, dim3(1), dim3(64), 0, s, gate, chunks, n);
    return hipGetLastError();
}

hipError_t launch_release_signal(uint64_t value_addr, hipStream_t s)
{
    if (!value_addr) return hipErrorInvalidValue;
    hipLaunchKernelGGL(release_signal_kernel, dim3(1), dim3(64), 0, s, reinterpret_cast<int64_t *>(value_addr));
    return hipGetLastError();
}

hipError_t launch_pack_weight(const uint16_t *W, uint16_t *Wt, int64_t K, int64_t N, hipStream_t s, uint32_t *clear, int clear_words)
{
    if (clear_words < 0 || clear_words > 256) return hipErrorInvalidValue;
    const unsigned tn = (unsigned)((N + 63) / 64);
    if ((uintptr_t)W % 16 == 0 && (uintptr_t)Wt % 16 == 0 && K % 64 == 0 && N % 8 == 0)
        hipLaunchKernelGGL(pack_weight_kernel, dim3(tn, (unsigned)((K + 255) / 256)), dim3(256), 0, s, W, Wt, K, N, clear, clear_words);
    else
        hipLaunchKernelGGL(pack_weight_unaligned_kernel, dim3(tn, (unsigned)((K + 63) / 64)), dim3(256), 0, s, W, Wt, K, N, clear, clear_words);
    return hipGetLastError();
}

hipError_t launch_grouped(int tile, const GroupedLaunch &r, hipStream_t s)
{
    switch (tile) {
#define X(id, T) case id: return launch_grouped_t<T>(r, s);
    FICCO_FOR_EACH_TILE(X)
#undef X
    default: return hipErrorInvalidValue;
    }
}

int grouped_grid_size(int tile, int device)
{
    switch (tile) {
#define X(id, T) case id: return grouped_grid_t<T>(device);
    FICCO_FOR_EACH_TILE(X)
#undef X
    default: return 0;
    }
}

}  // namespace ficco

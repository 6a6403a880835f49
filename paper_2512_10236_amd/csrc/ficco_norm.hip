// What stands between two blocks of a layer (ficco_residual_norm and its backward): norm behind a block, gate, scaled residual
// stream, norm in front of the next block. With D = width, r(v) = 1 / sqrt(mean(v^2) + eps):
//   n = p b r(b),  y = s x + g n,  h = w y r(y)
//   u = w dh,      dY = dy + r(y) (u - y r(y)^2 mean(u y)),  dx = s dY
//   dn = g dY,     db = r(b) (p dn - b r(b)^2 mean(p dn b)),  dg = sum dY n,  dp = sum dn b r(b),  dw = sum dh y r(y)
//
// Streaming work, bound by memory: a row lives in the registers of the threads that own it (V vectors of 8 values each)
// between its loads and its stores, and is read once. All sums are fp32.
#include "ficco_operators.h"
#include "ficco_epilogue.h"
#include "ficco_lanes.h"

namespace ficco {
namespace {

struct NormLaunch {
    const void *x;                // forward: x; backward: y
    const uint16_t *block;
    const void *post, *gate, *pre;
    void *y;                      // forward: y; backward: dx
    uint16_t *h;                  // forward: h; backward: dblock
    const void *dy;
    const uint16_t *dh;
    float *sum_post, *sum_gate, *sum_pre;      // backward: [chunks][width] partial sums (of one chunk: the sums), null: not wanted
    float *dgate;                 // backward: rows of dgate that a chunk holds whole groups of, else null
    int32_t rows, width, gate_rows, param_f32;
    int32_t chunks, per_group, chunk_rows;     // backward: chunk c is the (c % per_group)-th run of chunk_rows rows of its group, ...
                                               // ... or, with per_group 0, of all rows
    float scale, eps;
};

struct Vec8 {
    float f[8];
};
static __device__ __forceinline__ Vec8 widen(u32x4_t v)
{
    Vec8 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) { o.f[2 * i] = bf16_lo(v[i]); o.f[2 * i + 1] = bf16_hi(v[i]); }
    return o;
}
static __device__ __forceinline__ u32x4_t narrow(const Vec8 &v)
{
    return u32x4_t{pack2_bf16_rne(v.f[0], v.f[1]), pack2_bf16_rne(v.f[2], v.f[3]), pack2_bf16_rne(v.f[4], v.f[5]), pack2_bf16_rne(v.f[6], v.f[7])};
}
static __device__ __forceinline__ Vec8 from_f32x4(f32x4_t a, f32x4_t b)
{
    Vec8 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) { o.f[i] = a[i]; o.f[4 + i] = b[i]; }
    return o;
}
static __device__ __forceinline__ Vec8 from_f32(const float *p)
{
    return from_f32x4(reinterpret_cast<const f32x4_t *>(p)[0], reinterpret_cast<const f32x4_t *>(p)[1]);
}
// 8 values from element `at` (a multiple of 8) on, of either type
template <bool F32>
static __device__ __forceinline__ Vec8 load8(const void *p, int64_t at)
{
    if constexpr (F32) return from_f32(static_cast<const float *>(p) + at);
    else return widen(*reinterpret_cast<const u32x4_t *>(static_cast<const uint16_t *>(p) + at));
}
static __device__ __forceinline__ Vec8 param8(const void *p, int f32, int64_t at) { return f32 ? load8<true>(p, at) : load8<false>(p, at); }
template <bool F32>
static __device__ __forceinline__ void store8(void *p, int64_t at, const Vec8 &v)
{
    if constexpr (F32) {
        f32x4_t *o = reinterpret_cast<f32x4_t *>(static_cast<float *>(p) + at);
        o[0] = f32x4_t{v.f[0], v.f[1], v.f[2], v.f[3]};
        o[1] = f32x4_t{v.f[4], v.f[5], v.f[6], v.f[7]};
    } else {
        *reinterpret_cast<u32x4_t *>(static_cast<uint16_t *>(p) + at) = narrow(v);
    }
}

// TPR threads a row (a wavefront, with four rows a workgroup, or a whole workgroup), V vectors of 8 values a thread.
template <int TPR, int V>
struct RowCfg {
    static constexpr int THREADS = TPR == 64 ? 256 : TPR, ROWS = THREADS / TPR;
    static_assert(ROWS == 1 || TPR == 64, "a row's number is the same in a whole wavefront");
    static __device__ __forceinline__ int lane() { return ROWS == 1 ? threadIdx.x : threadIdx.x % 64; }
    static __device__ __forceinline__ int row() { return ROWS == 1 ? 0 : scalar(threadIdx.x / 64); }
};

// 2048 rows of 8192, the stream in fp32: 45 us, 4.5 TB/s, where a copy of 2 GiB reaches 4.9; eight rows 4 us, which are the way of a row
// from memory and its two sums.
template <int TPR, int V, bool F32>
__global__ __launch_bounds__((RowCfg<TPR, V>::THREADS)) void residual_norm_kernel(NormLaunch a)
{
    typedef RowCfg<TPR, V> R;
    constexpr int ROWS = R::ROWS;
    __shared__ float s_post[2][16], s_pre[2][16];
    const int lane = R::lane();
    const float inv = 1.0f / (float)a.width;
    const int vecs = a.width / 8;
    int turn = 0;                          // the sums' places in turns, so that they are not those a slower wavefront still reads
    for (int64_t row = (int64_t)blockIdx.x * ROWS + R::row(); row < a.rows; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const int64_t at = row * a.width;
        const int64_t gate_at = a.gate && a.gate_rows ? (int64_t)((int)row / a.gate_rows) * a.width : 0;
        u32x4_t b[V];
        Vec8 y[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = lane + v * TPR;
            b[v] = u32x4_t{0u, 0u, 0u, 0u};
            if (i < vecs) b[v] = *reinterpret_cast<const u32x4_t *>(a.block + at + i * 8);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = lane + v * TPR;
            y[v] = Vec8{};
            if (i < vecs) y[v] = load8<F32>(a.x, at + i * 8);
        }
        float r = 1.0f;
        if (a.post) {
            float ss[1] = {0.f};
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Vec8 w = widen(b[v]);
#pragma unroll
                for (int e = 0; e < 8; ++e) ss[0] = fmaf(w.f[e], w.f[e], ss[0]);
            }
            thread_sums<TPR, 1>(ss, s_post[turn]);
            r = rsqrtf(fmaf(ss[0], inv, a.eps));
        }
        float ss[1] = {0.f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = lane + v * TPR;
            if (i < vecs) {
                Vec8 n = widen(b[v]);
                if (a.post) {
                    const Vec8 p = param8(a.post, a.param_f32, i * 8);
#pragma unroll
                    for (int e = 0; e < 8; ++e) n.f[e] *= r * p.f[e];
                }
                if (a.gate) {
                    const Vec8 g = param8(a.gate, a.param_f32, gate_at + i * 8);
#pragma unroll
                    for (int e = 0; e < 8; ++e) n.f[e] *= g.f[e];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[v].f[e] = fmaf(a.scale, y[v].f[e], n.f[e]);
                    ss[0] = fmaf(y[v].f[e], y[v].f[e], ss[0]);
                }
                store8<F32>(a.y, at + i * 8, y[v]);
            }
        }
        if (a.h) {
            thread_sums<TPR, 1>(ss, s_pre[turn]);
            r = rsqrtf(fmaf(ss[0], inv, a.eps));
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int i = lane + v * TPR;
                if (i < vecs) {
                    const Vec8 w = param8(a.pre, a.param_f32, i * 8);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[v].f[e] *= r * w.f[e];
                    store8<false>(a.h, at + i * 8, y[v]);
                }
            }
        }
    }
}

// What a thread loads of a row for one vector, as it comes
template <bool F32>
struct RawRow {
    u32x4_t y[F32 ? 2 : 1], dy[F32 ? 2 : 1], b, dh;
};
template <bool F32>
static __device__ __forceinline__ void load_raw(u32x4_t (&r)[F32 ? 2 : 1], const void *p, int64_t at)
{
    const u32x4_t *v = reinterpret_cast<const u32x4_t *>(static_cast<const char *>(p) + at * (F32 ? 4 : 2));
    r[0] = __builtin_nontemporal_load(v);
    if constexpr (F32) r[1] = __builtin_nontemporal_load(v + 1);
}
template <bool F32>
static __device__ __forceinline__ Vec8 widen_raw(const u32x4_t (&r)[F32 ? 2 : 1])
{
    if constexpr (F32) {
        Vec8 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) { o.f[i] = __uint_as_float(r[0][i]); o.f[4 + i] = __uint_as_float(r[1][i]); }
        return o;
    } else return widen(r[0]);
}

// The backward's rows go in chunks, each walked by one group of TPR threads, which keeps its columns' partial sums in registers
// and writes them once: sums over rows in a fixed order, without atomics. A row needs two sums over its columns in turn, the
// second of what the first gives, so the next row is loaded before the first: its way from memory is then behind both. What a
// thread past the row's end loads is the row's first vector, and nothing comes of it. 16384 rows of 4096 in bf16, all gradients:
// 173 us with the sums, 4.7 TB/s.
template <int TPR, int V, bool F32>
__global__ __launch_bounds__((RowCfg<TPR, V>::THREADS), (V == 1 ? 4 : 2)) void residual_norm_backward_kernel(NormLaunch a)
{
    typedef RowCfg<TPR, V> R;
    constexpr int ROWS = R::ROWS;
    // One vector a thread: the parameters stay in 128 registers, and the next row is loaded early. Four, of longer rows: neither has
    // room in 256, and of the three partial sums two lie in LDS ([2][V][2][TPR] four floats each). 512 threads with four rather than
    // 1024 with two: what a thread has beside its values is there once for four, and nothing spills (3000 rows of 16384 in bf16
    // 162 us, 3.7 TB/s, against 179; one row 11 against 13). Narrower rows leave vectors of the four empty: of 12288 137 us, 3.2 TB/s, of 8200 116, 2.5.
    constexpr bool KEEP = V == 1;
    extern __shared__ f32x4_t s_acc[];
    __shared__ float s_a[2][3 * 16], s_b[2][16];      // in turns, so that a row's places are not those a slower wavefront still reads
    const int lane = R::lane(), chunk = blockIdx.x * ROWS + R::row();
    if (TPR == 64 && chunk >= a.chunks) return;
    const float inv = 1.0f / (float)a.width;
    const int vecs = a.width / 8;
    int64_t begin = (int64_t)chunk * a.chunk_rows, end = begin + a.chunk_rows;
    if (a.per_group) {
        const int g = chunk / a.per_group;
        begin = (int64_t)g * a.gate_rows + (int64_t)(chunk % a.per_group) * a.chunk_rows;
        end = min(begin + a.chunk_rows, (int64_t)(g + 1) * a.gate_rows);
    }
    end = min(end, (int64_t)a.rows);
    int col[V];
    float there[V];                        // 1, or 0 past the row's end
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const bool in = lane + v * TPR < vecs;
        col[v] = in ? (lane + v * TPR) * 8 : 0;
        there[v] = in ? 1.0f : 0.0f;
    }
    const bool has_dh = a.dh != nullptr, has_dy = a.dy != nullptr, has_b = a.block != nullptr, post = a.post != nullptr, gated = a.gate != nullptr;
    Vec8 kept_post{}, dgate[V], kept_pre{}, kept_w{}, kept_p{}, kept_g{};
#pragma unroll
    for (int v = 0; v < V; ++v) dgate[v] = Vec8{};
    auto place = [&](int which, int v, int half) __attribute__((always_inline)) { return s_acc + ((which * V + v) * 2 + half) * TPR + lane; };
    if constexpr (!KEEP)
#pragma unroll
        for (int k = 0; k < 4 * V; ++k) s_acc[k * TPR + lane] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // sum += t, of dpost (which = 0) or dpre (1): only this thread uses its places
    auto add = [&](Vec8 &kept, int which, int v, const Vec8 &t) __attribute__((always_inline)) {
        if constexpr (KEEP) {
#pragma unroll
            for (int e = 0; e < 8; ++e) kept.f[e] += t.f[e];
        } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x4_t s4 = *place(which, v, half);
#pragma unroll
                for (int e = 0; e < 4; ++e) s4[e] += t.f[4 * half + e];
                *place(which, v, half) = s4;
            }
        }
    };
    auto total = [&](const Vec8 &kept, int which, int v) __attribute__((always_inline)) {
        if constexpr (KEEP) return kept;
        else return from_f32x4(*place(which, v, 0), *place(which, v, 1));
    };
    if constexpr (KEEP) {
        if (has_dh) kept_w = param8(a.pre, a.param_f32, col[0]);
        if (post) kept_p = param8(a.post, a.param_f32, col[0]);
    }
    auto param = [&](const Vec8 &kept, const void *from, int64_t at) __attribute__((always_inline)) {
        if constexpr (KEEP) return kept;
        else {
            asm volatile("" : "+v"(at));   // not moved out of the loop over the rows
            return from ? param8(from, a.param_f32, at) : Vec8{};
        }
    };
    // without KEEP: one vector's values at a time
    auto apart = [&]() __attribute__((always_inline)) {
        if constexpr (!KEEP) __builtin_amdgcn_sched_barrier(0);
    };
    // ... and its values as they came, to be widened anew: else the compiler keeps them widened from one use to the next
    auto as_they_came = [&](RawRow<F32> &raw) __attribute__((always_inline)) {
        if constexpr (!KEEP) {
#pragma unroll
            for (int k = 0; k < (F32 ? 2 : 1); ++k) asm volatile("" : "+v"(raw.y[k]), "+v"(raw.dy[k]));
            asm volatile("" : "+v"(raw.b), "+v"(raw.dh));
        }
    };
    auto load = [&](RawRow<F32> &raw, int64_t row, int v) __attribute__((always_inline)) {
        const int64_t at = row * a.width + col[v];
        if (has_dh) {
            load_raw<F32>(raw.y, a.x, at);
            raw.dh = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(a.dh + at));
        }
        if (has_dy) load_raw<F32>(raw.dy, a.dy, at);
        if (has_b) raw.b = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(a.block + at));
    };
    RawRow<F32> next{};
    if (KEEP && begin < end) load(next, begin, 0);
    int group = a.gate_rows ? (int)(begin / a.gate_rows) : 0, group_end = a.gate_rows ? (int)min((int64_t)(group + 1) * a.gate_rows, (int64_t)a.rows) : a.rows;
    bool new_gate = true;
    for (int64_t row = begin; row < end; ++row) {
        const int64_t at = row * a.width;
        const int parity = (int)(row - begin) & 1;
        RawRow<F32> now[V];
        if constexpr (KEEP) now[0] = next;
        else
#pragma unroll
            for (int v = 0; v < V; ++v) {
                now[v] = RawRow<F32>{};
                load(now[v], row, v);
            }
        Vec8 d[V];                         // dy, then dY, then post * dn
        float s[3] = {0.f, 0.f, 0.f};      // y^2, u y, b^2
        if (KEEP && gated && new_gate) kept_g = param8(a.gate, a.param_f32, (int64_t)group * a.width + col[0]);
        new_gate = false;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Vec8 w = param(kept_w, has_dh ? a.pre : nullptr, col[v]);
            const Vec8 y = widen_raw<F32>(now[v].y), b = widen(now[v].b), dh = widen(now[v].dh);
            float t[3] = {0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                t[0] = fmaf(y.f[e], y.f[e], t[0]);
                t[1] = fmaf(w.f[e] * dh.f[e], y.f[e], t[1]);
                t[2] = fmaf(b.f[e], b.f[e], t[2]);
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) s[k] += there[v] != 0.f ? t[k] : 0.f;
            as_they_came(now[v]);
            apart();
        }
        if (KEEP && row + 1 < end) load(next, row + 1, 0);
        thread_sums<TPR, 3>(s, s_a[parity]);
        const float r = rsqrtf(fmaf(s[0], inv, a.eps)), back = r * (r * (r * s[1] * inv));   // r^3 alone may be past fp32's range
        const float rb = post ? rsqrtf(fmaf(s[2], inv, a.eps)) : 1.0f;
        float s4[1] = {0.f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const bool in = there[v] != 0.f;
            const Vec8 w = param(kept_w, has_dh ? a.pre : nullptr, col[v]), p = param(kept_p, a.post, col[v]);
            const Vec8 gt = param(kept_g, a.gate, (int64_t)group * a.width + col[v]);
            d[v] = widen_raw<F32>(now[v].dy);
            const Vec8 b = widen(now[v].b);
            if (has_dh) {
                const Vec8 y = widen_raw<F32>(now[v].y), dh = widen(now[v].dh);
                Vec8 t;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    d[v].f[e] += fmaf(r * w.f[e], dh.f[e], -y.f[e] * back);
                    t.f[e] = dh.f[e] * r * y.f[e];
                }
                add(kept_pre, 1, v, t);
            }
            if (a.y && in) {
                Vec8 o;
#pragma unroll
                for (int e = 0; e < 8; ++e) o.f[e] = a.scale * d[v].f[e];
                store8<F32>(a.y, at + col[v], o);
            }
            if (gated) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float n = post ? b.f[e] * rb * p.f[e] : b.f[e];
                    dgate[v].f[e] = fmaf(d[v].f[e], n, dgate[v].f[e]);
                    d[v].f[e] *= gt.f[e];
                }
            }
            if (post) {
                float sum = 0.f;
                Vec8 t;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    t.f[e] = d[v].f[e] * (b.f[e] * rb);
                    d[v].f[e] *= p.f[e];
                    sum = fmaf(d[v].f[e], b.f[e], sum);
                }
                s4[0] += in ? sum : 0.f;
                add(kept_post, 0, v, t);
            }
            as_they_came(now[v]);
            apart();
        }
        if (post) thread_sums<TPR, 1>(s4, s_b[parity]);
        if (a.h) {
            const float back_b = rb * (rb * (rb * s4[0] * inv));
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (post) {
                    const Vec8 b = widen(now[v].b);
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[v].f[e] = fmaf(rb, d[v].f[e], -b.f[e] * back_b);
                }
                if (there[v] != 0.f) store8<false>(a.h, at + col[v], d[v]);
                apart();
            }
        }
        if (row + 1 == group_end && a.gate_rows) {
            // a group of rows that share a gate ends; where a chunk holds whole groups it writes their sums
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (a.dgate) {
                    if (there[v] != 0.f) store8<true>(a.dgate, (int64_t)group * a.width + col[v], dgate[v]);
                    dgate[v] = Vec8{};
                }
            }
            ++group;
            group_end = (int)min((int64_t)group_end + a.gate_rows, (int64_t)a.rows);
            new_gate = true;
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (there[v] != 0.f) {
            const int64_t at = (int64_t)chunk * a.width + col[v];
            if (a.sum_post) store8<true>(a.sum_post, at, total(kept_post, 0, v));
            if (a.sum_gate) store8<true>(a.sum_gate, at, dgate[v]);
            if (a.sum_pre) store8<true>(a.sum_pre, at, total(kept_pre, 1, v));
        }
    }
}

// Sums of the chunks' partial sums, 32 columns a workgroup. blockIdx.y = 0: dpost over all chunks, 1: dpre, 2 + g: dgate of group
// g over its own chunks.
struct SumLaunch {
    const float *sums;
    float *dpost, *dgate, *dpre;
    int32_t chunks, per_group, width;
};
__global__ __launch_bounds__(1024) void residual_norm_sum_kernel(SumLaunch a)
{
    __shared__ float s[32][32];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31);
    const int64_t plane = (int64_t)a.chunks * a.width;
    const int y = blockIdx.y;
    const float *in = y == 0 ? a.sums : y == 1 ? a.sums + 2 * plane : a.sums + plane + (int64_t)(y - 2) * a.per_group * a.width;
    float *out = y == 0 ? a.dpost : y == 1 ? a.dpre : a.dgate ? a.dgate + (int64_t)(y - 2) * a.width : nullptr;
    if (!out) return;
    const float t = column_sum(in + c, y < 2 ? a.chunks : a.per_group, a.width, c < a.width, s);
    if (threadIdx.x < 32 && c < a.width) out[c] = t;
}

// ------------------------------------------------------------------------------------------------------------- host
int checked(const ficco_residual_norm_t *op, ficco_residual_norm_t *out)
{
    if (!op) return FICCO_ERR_ARG;
    const ficco_residual_norm_t &o = *op;
    if (o.stream_type < FICCO_BF16 || o.stream_type > FICCO_F32 || o.param_type < FICCO_BF16 || o.param_type > FICCO_F32) return FICCO_ERR_ARG;
    if (!(o.eps >= 0.f) || !std::isfinite(o.eps) || !std::isfinite(o.residual_scale)) return FICCO_ERR_ARG;
    if (o.rows < 0 || o.rows > 0x7FFFFFFF || o.width < 8 || o.width % 8 || o.width > 16384 || o.gate_rows < 0) return FICCO_ERR_SHAPE;
    *out = o;
    if (out->gate_rows > std::max<int64_t>(o.rows, 1)) out->gate_rows = std::max<int64_t>(o.rows, 1);
    return FICCO_OK;
}

// Threads a row: one vector a thread, as far as a workgroup's 1024 threads go.
int threads_of(int64_t width)
{
    for (int tpr : {64, 128, 192, 256, 384, 512, 768})
        if (width <= tpr * 8) return tpr;
    return 1024;
}

struct Chunks {
    int64_t chunks, per_group, rows, groups;
    bool whole_groups;            // a chunk holds whole groups: it writes their dgate itself
};
Chunks chunks_of(const ficco_residual_norm_t &o)
{
    // as many as run at once on 256 CUs with 1024 threads each; but a chunk's sums are written and read again, so more than 1024 of
    // them only where each has 16 rows
    const int64_t most = 256 * 1024 / threads_of(o.width);
    const int64_t target = std::min(most, std::max<int64_t>(1024, o.rows / 16));
    int64_t each = std::max<int64_t>(1, (o.rows + target - 1) / target);
    // three rows or fewer in one chunk need no second launch (3 rows of 960, replayed and called: 5.7 and 6.6 us, in chunks of one
    // 5.6 and 9.0; 4 rows 7.0 and 7.0, 5.6 and 9.1; 3 rows of 7192 11.0, 9.7)
    if (o.rows <= 3 && o.width <= 4096) each = std::max<int64_t>(1, o.rows);
    Chunks c{};
    if (!o.gate_rows || o.gate_rows >= o.rows) {
        c.groups = 1;
        c.rows = each;
        c.chunks = c.per_group = (o.rows + each - 1) / each;
    } else if (o.gate_rows >= each) {
        c.groups = (o.rows + o.gate_rows - 1) / o.gate_rows;
        c.per_group = (o.gate_rows + each - 1) / each;
        c.rows = (o.gate_rows + c.per_group - 1) / c.per_group;
        c.chunks = c.groups * c.per_group;
    } else {
        c.whole_groups = true;
        c.rows = each / o.gate_rows * o.gate_rows;
        c.chunks = (o.rows + c.rows - 1) / c.rows;
    }
    return c;
}
int64_t workspace_of(const ficco_residual_norm_t &o) { return o.rows ? 3 * chunks_of(o).chunks * o.width * 4 : 0; }

template <int TPR, int V>
int launch_forward_t(const NormLaunch &a, bool f32, hipStream_t s)
{
    typedef RowCfg<TPR, V> R;
    const dim3 grid((unsigned)std::min<int64_t>(((int64_t)a.rows + R::ROWS - 1) / R::ROWS, 1 << 20)), block(R::THREADS);
    if (f32) hipLaunchKernelGGL((residual_norm_kernel<TPR, V, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((residual_norm_kernel<TPR, V, false>), grid, block, 0, s, a);
    HIP_TRY(hipGetLastError());
    return FICCO_OK;
}

int launch_forward(const NormLaunch &a, bool f32, hipStream_t s)
{
    switch (threads_of(a.width)) {
    case 64: return launch_forward_t<64, 1>(a, f32, s);
    case 128: return launch_forward_t<128, 1>(a, f32, s);
    case 192: return launch_forward_t<192, 1>(a, f32, s);
    case 256: return launch_forward_t<256, 1>(a, f32, s);
    case 384: return launch_forward_t<384, 1>(a, f32, s);
    case 512: return launch_forward_t<512, 1>(a, f32, s);
    case 768: return launch_forward_t<768, 1>(a, f32, s);
    }
    return a.width <= 8192 ? launch_forward_t<1024, 1>(a, f32, s) : launch_forward_t<1024, 2>(a, f32, s);
}

template <int TPR, int V>
int launch_backward_t(const NormLaunch &a, bool f32, hipStream_t s)
{
    typedef RowCfg<TPR, V> R;
    const dim3 grid((unsigned)((a.chunks + R::ROWS - 1) / R::ROWS)), block(R::THREADS);
    constexpr int LDS = V == 1 ? 0 : 2 * V * 2 * TPR * 16;
    const auto fn = f32 ? &residual_norm_backward_kernel<TPR, V, true> : &residual_norm_backward_kernel<TPR, V, false>;
    if (LDS) HIP_TRY((f32 ? raise_lds_limit<&residual_norm_backward_kernel<TPR, V, true>>(LDS) : raise_lds_limit<&residual_norm_backward_kernel<TPR, V, false>>(LDS)));
    hipLaunchKernelGGL(fn, grid, block, LDS, s, a);
    HIP_TRY(hipGetLastError());
    return FICCO_OK;
}

int launch_backward(const NormLaunch &a, bool f32, hipStream_t s)
{
    switch (threads_of(a.width)) {
    case 64: return launch_backward_t<64, 1>(a, f32, s);
    case 128: return launch_backward_t<128, 1>(a, f32, s);
    case 192: return launch_backward_t<192, 1>(a, f32, s);
    case 256: return launch_backward_t<256, 1>(a, f32, s);
    case 384: return launch_backward_t<384, 1>(a, f32, s);
    case 512: return launch_backward_t<512, 1>(a, f32, s);
    case 768: return launch_backward_t<768, 1>(a, f32, s);
    }
    return a.width <= 8192 ? launch_backward_t<1024, 1>(a, f32, s) : launch_backward_t<512, 4>(a, f32, s);
}

int forward(const ficco_residual_norm_t *op, const void *x, const void *block, const void *post, const void *gate, const void *pre, void *y, void *h,
            hipStream_t s)
{
    ficco_residual_norm_t o;
    int rc = checked(op, &o);
    if (rc) return rc;
    const bool none = o.rows == 0;
    if (!pre != !h) return FICCO_ERR_ARG;
    rc = check_args({{x, 16, none}, {block, 16, none}, {post, 16, true}, {gate, 16, true}, {pre, 16, true}, {y, 16, none}, {h, 16, true}});
    if (rc || none) return rc;
    NormLaunch a{};
    a.x = x; a.block = (const uint16_t *)block; a.post = post; a.gate = gate; a.pre = pre; a.y = y; a.h = (uint16_t *)h;
    a.rows = (int32_t)o.rows; a.width = (int32_t)o.width; a.gate_rows = (int32_t)o.gate_rows;
    a.param_f32 = o.param_type == FICCO_F32;
    a.scale = o.residual_scale; a.eps = o.eps;
    return launch_forward(a, o.stream_type == FICCO_F32, s);
}

int backward(const ficco_residual_norm_t *op, const void *y, const void *block, const void *post, const void *gate, const void *pre, const void *dy,
             const void *dh, void *dx, void *dblock, void *dpost, void *dgate, void *dpre, void *workspace, int64_t workspace_bytes, hipStream_t s)
{
    ficco_residual_norm_t o;
    int rc = checked(op, &o);
    if (rc) return rc;
    const bool none = o.rows == 0, sums = dpost || dgate || dpre;
    if ((dpost && !post) || (dgate && !gate) || (dpre && !pre) || (dpre && !dh && !none) || (dh && !pre)) return FICCO_ERR_ARG;
    const bool needs_block = dpost || dgate || (dblock && post);
    rc = check_args({{y, 16, none || !dh}, {block, 16, none || !needs_block}, {post, 16, true}, {gate, 16, true}, {pre, 16, true}, {dy, 16, true}, {dh, 16, true},
                     {dx, 16, true}, {dblock, 16, true}, {dpost, 16, true}, {dgate, 16, true}, {dpre, 16, true}, {workspace, 16, none || !sums}});
    if (rc) return rc;
    if (sums && workspace_bytes < workspace_of(o)) return FICCO_ERR_ARG;
    if (!dx && !dblock && !sums) return FICCO_OK;
    const Chunks c = chunks_of(o);
    const bool one = c.chunks == 1;        // its sums are the sums
    SumLaunch t{(const float *)workspace, (float *)dpost, nullptr, (float *)dpre, (int32_t)c.chunks, (int32_t)c.per_group, (int32_t)o.width};
    int groups = 0;
    if (dgate && !c.whole_groups && (!none || !op->gate_rows)) { t.dgate = (float *)dgate; groups = (int)c.groups; }
    if (!none) {
        NormLaunch a{};
        a.x = y; a.block = needs_block ? (const uint16_t *)block : nullptr; a.post = needs_block ? post : nullptr; a.gate = gate; a.pre = pre;
        a.y = dx; a.h = (uint16_t *)dblock; a.dy = dy; a.dh = (const uint16_t *)dh;
        const int64_t plane = c.chunks * o.width;
        float *const ws = (float *)workspace;
        a.sum_post = one || !dpost ? (float *)dpost : ws;
        a.sum_gate = c.whole_groups ? nullptr : one || !dgate ? (float *)dgate : ws + plane;
        a.sum_pre = one || !dpre ? (float *)dpre : ws + 2 * plane;
        a.dgate = c.whole_groups ? (float *)dgate : nullptr;
        a.rows = (int32_t)o.rows; a.width = (int32_t)o.width; a.gate_rows = (int32_t)o.gate_rows;
        a.param_f32 = o.param_type == FICCO_F32;
        a.chunks = (int32_t)c.chunks; a.chunk_rows = (int32_t)c.rows;
        a.per_group = c.groups > 1 ? (int32_t)c.per_group : 0;
        a.scale = o.residual_scale; a.eps = o.eps;
        if ((rc = launch_backward(a, o.stream_type == FICCO_F32, s))) return rc;
    }
    if (!one && (dpost || dpre || t.dgate)) {
        hipLaunchKernelGGL(residual_norm_sum_kernel, dim3((unsigned)((o.width + 31) / 32), (unsigned)(2 + groups)), dim3(1024), 0, s, t);
        HIP_TRY(hipGetLastError());
    }
    return FICCO_OK;
}

}  // namespace
}  // namespace ficco

using namespace ficco;

extern "C" {

int ficco_residual_norm_workspace(const ficco_residual_norm_t *op, int64_t *bytes)
{
    return guarded([&] {
        ficco_residual_norm_t o;
        if (!bytes) return (int)FICCO_ERR_ARG;
        const int rc = checked(op, &o);
        if (rc) return rc;
        *bytes = workspace_of(o);
        return (int)FICCO_OK;
    });
}

int ficco_residual_norm(const ficco_residual_norm_t *op, const void *x, const void *block, const void *post_weight, const void *gate,
                        const void *pre_weight, void *y, void *h, void *stream)
{
    return guarded([&] { return forward(op, x, block, post_weight, gate, pre_weight, y, h, (hipStream_t)stream); });
}

int ficco_residual_norm_backward(const ficco_residual_norm_t *op, const void *y, const void *block, const void *post_weight, const void *gate,
                                 const void *pre_weight, const void *dy, const void *dh, void *dx, void *dblock, void *dpost_weight, void *dgate,
                                 void *dpre_weight, void *workspace, int64_t workspace_bytes, void *stream)
{
    return guarded([&] {
        return backward(op, y, block, post_weight, gate, pre_weight, dy, dh, dx, dblock, dpost_weight, dgate, dpre_weight, workspace, workspace_bytes,
                        (hipStream_t)stream);
    });
}

}  // extern "C"

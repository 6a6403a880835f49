// Counts of tokens per expert and the balance loss of a router (ficco_expert_balance and its backward). For a group g of tokens
// with n valid ones, c_e slots of which went to expert e, and p_t = softmax(logits_t):
//   loss = sum over g of s sum_e c_e sum_t p_te,   s = coefficient E / (G k n^2)
//   d loss / d logits_te = s p_te (c_e - sum_j c_j p_tj)
// Streaming work over the logits; a group of lanes has a token, V of its logits a lane. Column sums stay in registers and go to
// memory once per chunk of tokens, so that all sums have a fixed order; counts are integers. The gradient's difference is small
// next to its parts where a router is nearly even, so it is taken of the counts' distances from their mean, which are exact.
#include "ficco_operators.h"
#include "ficco_epilogue.h"
#include "ficco_lanes.h"
#include "ficco_token_run.h"

namespace ficco {
namespace {

struct BalanceLaunch {
    const void *logits;
    const int32_t *ids;
    const uint8_t *valid;
    int32_t *counts, *group_valid;
    float *loss;
    const float *dloss;
    void *dlogits;
    // partial results of a chunk of tokens, where a group has several: [chunks][E], [chunks][E], [chunks]
    float *part_p;
    int32_t *part_c, *part_n;
    float *terms;                 // [n_terms] parts of the loss: of the groups, or of 64 experts of a group each (one: the loss itself)
    int32_t n_terms;
    int64_t ld;
    int32_t tokens, group_tokens, groups, experts, top_k;
    int32_t per_group, chunk_tokens;       // see token_run
    float coefficient;
};

static __device__ __forceinline__ float logit(const float *p) { return *p; }
static __device__ __forceinline__ float logit(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
static __device__ __forceinline__ void put(float *p, float v) { *p = v; }
static __device__ __forceinline__ void put(uint16_t *p, float v) { *p = (uint16_t)pack2_bf16_rne(v, 0.f); }
// Four logits in one access, from any address that one of them may have: the memory path takes such accesses, and where they cross a
// line they take no longer (65536 x 256 with both directions, off by one logit: 51.9 us in fp32 and 53.6 in bf16, aligned 52.3 and 54.5)
typedef f32x4_t four_f32 __attribute__((aligned(4)));
typedef uint32_t four_bf16 __attribute__((ext_vector_type(2), aligned(2)));
static __device__ __forceinline__ f32x4_t logit4(const float *p) { return *reinterpret_cast<const four_f32 *>(p); }
static __device__ __forceinline__ f32x4_t logit4(const uint16_t *p)
{
    const four_bf16 v = *reinterpret_cast<const four_bf16 *>(p);
    return f32x4_t{bf16_lo(v[0]), bf16_hi(v[0]), bf16_lo(v[1]), bf16_hi(v[1])};
}
static __device__ __forceinline__ void put4(float *p, f32x4_t v) { *reinterpret_cast<four_f32 *>(p) = v; }
static __device__ __forceinline__ void put4(uint16_t *p, f32x4_t v) { *reinterpret_cast<four_bf16 *>(p) = four_bf16{pack2_bf16_rne(v[0], v[1]), pack2_bf16_rne(v[2], v[3])}; }

// A token's logits over LANES lanes, V each. Lane l has the experts l, l + LANES, ...; or, with FOURS (V a multiple of 4, rows of
// whole fours), the fours l, l + LANES, ... Which of the two follows from the sizes alone, since the order of a row's sums goes with it.
template <int LANES, int V, bool FOURS>
struct Spread {
    static constexpr int TOKENS = V <= 4 ? 4 : V <= 8 ? 2 : 1;     // tokens that a lane loads before it uses the first
    static __device__ __forceinline__ int expert(int lane, int v) { return FOURS ? 4 * (lane + v / 4 * LANES) + v % 4 : lane + v * LANES; }
    template <class L>
    static __device__ __forceinline__ void load(float (&x)[V], const L *row, int lane, int E)
    {
        if constexpr (FOURS) {
#pragma unroll
            for (int q = 0; q < V / 4; ++q)
                if (expert(lane, 4 * q) < E) {
                    const f32x4_t f = logit4(row + expert(lane, 4 * q));
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[4 * q + i] = f[i];
                }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (expert(lane, v) < E) x[v] = logit(row + expert(lane, v));
        }
    }
    template <class L>
    static __device__ __forceinline__ void store(const float (&x)[V], L *row, int lane, int E)
    {
        if constexpr (FOURS) {
#pragma unroll
            for (int q = 0; q < V / 4; ++q)
                if (expert(lane, 4 * q) < E) put4(row + expert(lane, 4 * q), f32x4_t{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]});
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (expert(lane, v) < E) put(row + expert(lane, v), x[v]);
        }
    }
};

// s of a group with n valid tokens
static __device__ __forceinline__ float group_scale(const BalanceLaunch &a, int n)
{
    return n > 0 ? a.coefficient * (float)a.experts / ((float)a.groups * (float)a.top_k * (float)n * (float)n) : 0.f;
}

static __device__ __forceinline__ TokenRun chunk_run(const BalanceLaunch &a, int chunk)
{
    return token_run(chunk, a.per_group, a.chunk_tokens, a.group_tokens, a.tokens);
}

// The probabilities of a token, in place of its logits. A token whose logits are all -inf has none.
template <int LANES, int V>
static __device__ __forceinline__ void softmax(float (&x)[V])
{
    float m = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) m = fmaxf(m, x[v]);
    m = lane_max<LANES>(m);
    if (m == -INFINITY) m = 0.f;
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        x[v] = __builtin_amdgcn_exp2f((x[v] - m) * kLog2E);
        s += x[v];
    }
    s = lane_sum<LANES>(s);
    const float r = s == 0.f ? 0.f : 1.0f / s;
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] *= r;
}

// Calls f(token, probabilities) for the tokens of a workgroup's run, LANES lanes a token and TOKENS of them at a time, so that their
// loads are in flight together. Padding, and what is behind the end, has no probabilities; its logits are not read.
template <class L, int LANES, int V, bool FOURS, class Fn>
static __device__ __forceinline__ void for_tokens(const BalanceLaunch &a, const TokenRun &run, Fn &&f)
{
    typedef Spread<LANES, V, FOURS> S;
    constexpr int SUBS = 256 / LANES, T = S::TOKENS;
    const int lane = threadIdx.x % LANES, sub = LANES == 64 ? scalar(threadIdx.x / 64) : threadIdx.x / LANES;
    const L *logits = static_cast<const L *>(a.logits);
    const int64_t end = run.end;
    int64_t first = run.begin + sub;
    int use[T];
    auto look = [&](int64_t t0) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < T; ++k) {
            const int64_t t = t0 + k * SUBS;
            use[k] = t < end;
            if (a.valid && t < end) use[k] = a.valid[t];
        }
    };
    look(first);
    for (; first < end; first += T * SUBS) {
        float x[T][V];
#pragma unroll
        for (int k = 0; k < T; ++k) {
#pragma unroll
            for (int v = 0; v < V; ++v) x[k][v] = -INFINITY;
            if (LANES == 64 ? scalar(use[k]) : use[k]) S::load(x[k], logits + (first + k * SUBS) * a.ld, lane, a.experts);
        }
        look(first + T * SUBS);
#pragma unroll
        for (int k = 0; k < T; ++k) softmax<LANES, V>(x[k]);
#pragma unroll
        for (int k = 0; k < T; ++k) f(first + k * SUBS, x[k]);
    }
}

// Sum over a workgroup of 4 wavefronts (256 threads) or 16, in a fixed order; thread 0 has it.
static __device__ __forceinline__ float workgroup_sum(float v, float *s)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = 0.f;
    if (threadIdx.x == 0)
        for (int w = 0; w < (int)blockDim.x / 64; ++w) t += s[w];
    return t;
}

// 65536 x 256 logits in fp32, 16 groups, top 8: 21 us with the join, of which the logits are 14 at a copy's rate; the slots' counters in LDS
// and the chunk's end are the rest.
// One chunk of tokens a workgroup. Where a group is one chunk (per_group == 1) it writes the group's results.
template <class L, int LANES, int V, bool FOURS>
__global__ __launch_bounds__(256) void balance_kernel(BalanceLaunch a)
{
    typedef Spread<LANES, V, FOURS> S;
    constexpr int SUBS = 256 / LANES;
    extern __shared__ float s_p[];         // [SUBS][LANES * V], then the chunk's counts
    __shared__ float s_sum[4];
    __shared__ int s_n;
    int *const s_c = reinterpret_cast<int *>(s_p + SUBS * LANES * V);
    const int E = a.experts;
    const TokenRun run = chunk_run(a, blockIdx.x);
    const int group = run.group;
    for (int e = threadIdx.x; e < E; e += 256) s_c[e] = 0;
    if (threadIdx.x == 0) s_n = 0;
    __syncthreads();
    for (int64_t i = run.begin * a.top_k + threadIdx.x; i < run.end * a.top_k; i += 256) {
        const int id = a.ids[i];
        if ((unsigned)id < (unsigned)E && (!a.valid || a.valid[i / a.top_k])) atomicAdd(s_c + id, 1);
    }
    if (a.valid) {
        int n = 0;
        for (int64_t t = run.begin + threadIdx.x; t < run.end; t += 256) n += a.valid[t] != 0;
        if (n) atomicAdd(&s_n, n);
    }
    if (a.loss) {
        const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
        float p[V];
#pragma unroll
        for (int v = 0; v < V; ++v) p[v] = 0.f;
        for_tokens<L, LANES, V, FOURS>(a, run, [&](int64_t, const float (&x)[V]) __attribute__((always_inline)) {
#pragma unroll
            for (int v = 0; v < V; ++v) p[v] += x[v];
        });
#pragma unroll
        for (int v = 0; v < V; ++v) s_p[sub * LANES * V + S::expert(lane, v)] = p[v];
    }
    __syncthreads();
    const int n = a.valid ? s_n : (int)(run.end - run.begin);
    float term = 0.f;
    for (int e = threadIdx.x; e < E; e += 256) {
        float t = 0.f;
        if (a.loss)
            for (int s = 0; s < SUBS; ++s) t += s_p[s * LANES * V + e];
        if (a.per_group == 1) {
            a.counts[(int64_t)group * E + e] = s_c[e];
            term += (float)s_c[e] * t;
        } else {
            a.part_c[(int64_t)blockIdx.x * E + e] = s_c[e];
            if (a.loss) a.part_p[(int64_t)blockIdx.x * E + e] = t;
        }
    }
    if (a.per_group == 1) {
        if (threadIdx.x == 0) a.group_valid[group] = n;
        if (a.loss) {
            const float sum = workgroup_sum(term, s_sum);
            if (threadIdx.x == 0) (a.n_terms == 1 ? a.loss : a.terms + group)[0] = sum * group_scale(a, n);
        }
    } else if (threadIdx.x == 0) {
        a.part_n[blockIdx.x] = n;
    }
}

// The chunks' results of group blockIdx.x for 64 experts from 64 blockIdx.y on, and 64 gridDim.y further, ...; 16 wavefronts take every
// 16th chunk, eight of theirs at a time (a chunk that is not there: the last, of which nothing is added).
__global__ __launch_bounds__(1024) void balance_group_kernel(BalanceLaunch a)
{
    __shared__ float s_p[16][64];
    __shared__ int s_c[16][64], s_n;
    const int E = a.experts, group = blockIdx.x, lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6);
    if (threadIdx.x == 0) s_n = 0;
    __syncthreads();
    int n = 0;
    for (int c = threadIdx.x; c < a.per_group; c += 1024) n += a.part_n[group * a.per_group + c];
    if (n) atomicAdd(&s_n, n);
    float term = 0.f;
    for (int slab = blockIdx.y; slab * 64 < E; slab += gridDim.y) {
        const int e = slab * 64 + lane;
        const int64_t first = (int64_t)group * a.per_group * E + min(e, E - 1);
        float t = 0.f;
        int count = 0;
        for (int c = wave; c < a.per_group; c += 128) {
            int pc[8];
            float pt[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int64_t at = first + (int64_t)min(c + 16 * k, a.per_group - 1) * E;
                pc[k] = a.part_c[at];
                pt[k] = a.loss ? a.part_p[at] : 0.f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + 16 * k < a.per_group) { count += pc[k]; t += pt[k]; }
        }
        __syncthreads();                   // the slab before is done with
        s_p[wave][lane] = t;
        s_c[wave][lane] = count;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int k = 1; k < 16; ++k) { t += s_p[k][lane]; count += s_c[k][lane]; }
            if (e < E) {
                a.counts[(int64_t)group * E + e] = count;
                term += (float)count * t;
            }
        }
    }
    if (wave) return;
    if (threadIdx.x == 0 && blockIdx.y == 0) a.group_valid[group] = s_n;
    if (a.loss) {
        const float sum = lane_sum<64>(term);
        if (threadIdx.x == 0) (a.n_terms == 1 ? a.loss : a.terms + (int64_t)group * gridDim.y + blockIdx.y)[0] = sum * group_scale(a, s_n);
    }
}

// loss = sum of the groups' parts (none: 0)
__global__ __launch_bounds__(1024) void balance_loss_kernel(const float *terms, int n, float *loss)
{
    __shared__ float s[16];
    float t = 0.f;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += 1024) t += terms[i];
    const float sum = workgroup_sum(t, s);
    if (threadIdx.x == 0) loss[0] = sum;
}

// 65536 x 256 in fp32: 23 us, 5.8 TB/s where the forward has just read the logits.
template <class L, int LANES, int V, bool FOURS>
__global__ __launch_bounds__(256) void balance_backward_kernel(BalanceLaunch a)
{
    typedef Spread<LANES, V, FOURS> S;
    const int E = a.experts, lane = threadIdx.x % LANES;
    const TokenRun run = chunk_run(a, blockIdx.x);
    const int group = run.group;
    int c[V], total = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        c[v] = S::expert(lane, v) < E ? a.counts[(int64_t)group * E + S::expert(lane, v)] : 0;
        total += c[v];
    }
#pragma unroll
    for (int d = LANES / 2; d >= 1; d >>= 1) total += __shfl_xor(total, d, 64);
    // experts times the distance from the mean, a whole number
    float dist[V];
#pragma unroll
    for (int v = 0; v < V; ++v) dist[v] = (float)((int64_t)c[v] * E - total);
    const float scale = group_scale(a, a.group_valid[group]) / (float)E * (a.dloss ? a.dloss[0] : 1.0f);
    L *dlogits = static_cast<L *>(a.dlogits);
    for_tokens<L, LANES, V, FOURS>(a, run, [&](int64_t t, const float (&x)[V]) __attribute__((always_inline)) {
        float mean = 0.f, d[V];
#pragma unroll
        for (int v = 0; v < V; ++v) mean = fmaf(x[v], dist[v], mean);
        mean = lane_sum<LANES>(mean);
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = scale * x[v] * (dist[v] - mean);
        if (t < run.end) S::store(d, dlogits + t * a.ld, lane, E);
    });
}

// ------------------------------------------------------------------------------------------------------------- host
int checked(const ficco_expert_balance_t *op, ficco_expert_balance_t *out)
{
    if (!op) return FICCO_ERR_ARG;
    ficco_expert_balance_t o = *op;
    if (o.logits_type < FICCO_BF16 || o.logits_type > FICCO_F32 || !std::isfinite(o.coefficient)) return FICCO_ERR_ARG;
    if (o.tokens < 0 || o.tokens > 0x7FFFFFFF || o.experts < 1 || o.experts > 1024 || o.top_k < 1 || o.top_k > 64 || o.group_tokens < 0) return FICCO_ERR_SHAPE;
    if (!o.group_tokens || o.group_tokens > o.tokens) o.group_tokens = std::max<int64_t>(o.tokens, 1);
    if (o.group_tokens * o.top_k > 0x7FFFFFFF) return FICCO_ERR_SHAPE;       // a count's 32 bits
    if ((o.tokens + o.group_tokens - 1) / o.group_tokens > (1 << 20)) return FICCO_ERR_SHAPE;
    if (!o.ld_logits) o.ld_logits = o.experts;
    if (o.ld_logits < o.experts || o.ld_logits > kMaxK) return FICCO_ERR_SHAPE;
    *out = o;
    return FICCO_OK;
}

int lanes_of(int experts) { return experts <= 8 ? 8 : experts <= 16 ? 16 : experts <= 32 ? 32 : 64; }

struct Chunks {
    int64_t groups, per_group, tokens, joins;      // joins: workgroups that join a group's chunks
};
void cut(const ficco_expert_balance_t &o, Chunks &c, int64_t per_group)
{
    c.per_group = std::max<int64_t>(1, std::min(per_group, o.group_tokens));
    c.tokens = (o.group_tokens + c.per_group - 1) / c.per_group;
}
// A group whose tokens a workgroup takes in 24 turns or fewer is one chunk, which spares the launches that join them. Else the time
// is that of a chunk's turns and, for the join, that of the number of chunks: least at the root of their product, up to four
// workgroups a CU of 256 CUs. us (tokens x experts, chunks of one group): 41825 x 22 64 31.2, 256 14.5, 512 13.1, 1024 19.3; 3000 x 64 32 14.1,
// 128 10.5, 512 12.0; 65536 x 256 256 31.6, 512 25.3, 1024 29.7.
Chunks forward_chunks(const ficco_expert_balance_t &o)
{
    Chunks c{};
    c.groups = (o.tokens + o.group_tokens - 1) / o.group_tokens;
    const int64_t turn = 256 / lanes_of(o.experts), turns = (o.group_tokens + turn - 1) / turn;
    cut(o, c, turns <= 24 ? 1 : std::min((int64_t)sqrt(24.0 * (double)turns), std::max<int64_t>(1, 1024 / c.groups)));
    c.joins = c.groups == 1 && o.experts <= 256 && c.per_group <= 128 ? 1 : (o.experts + 63) / 64;      // one: no launch for the loss
    return c;
}
// The backward joins nothing: about four workgroups a CU of 256 CUs.
Chunks backward_chunks(const ficco_expert_balance_t &o)
{
    Chunks c{};
    c.groups = (o.tokens + o.group_tokens - 1) / o.group_tokens;
    const int64_t each = std::max((o.tokens + 1023) / 1024, (int64_t)256 / lanes_of(o.experts));
    cut(o, c, (o.group_tokens + each - 1) / each);
    return c;
}

struct Workspace {
    int64_t p, c, n, terms, n_terms, bytes;
};
Workspace workspace_of(const ficco_expert_balance_t &o)
{
    const Chunks c = forward_chunks(o);
    Workspace w{};
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    if (c.per_group > 1) {
        w.p = take(c.groups * c.per_group * o.experts * 4);
        w.c = take(c.groups * c.per_group * o.experts * 4);
        w.n = take(c.groups * c.per_group * 4);
    }
    w.n_terms = c.groups * (c.per_group > 1 ? c.joins : 1);
    if (w.n_terms > 1) w.terms = take(w.n_terms * 4);
    w.bytes = at;
    return w;
}

BalanceLaunch launch_of(const ficco_expert_balance_t &o, const Chunks &c)
{
    BalanceLaunch a{};
    a.ld = o.ld_logits;
    a.tokens = (int32_t)o.tokens;
    a.group_tokens = (int32_t)o.group_tokens;
    a.groups = (int32_t)c.groups;
    a.experts = o.experts;
    a.top_k = o.top_k;
    a.per_group = (int32_t)c.per_group;
    a.chunk_tokens = (int32_t)c.tokens;
    a.coefficient = o.coefficient;
    return a;
}

template <class L, int LANES, int V, bool FOURS>
int launch_t(const BalanceLaunch &a, bool backward, hipStream_t s)
{
    const dim3 grid((unsigned)(a.groups * a.per_group)), block(256);
    if (backward) hipLaunchKernelGGL((balance_backward_kernel<L, LANES, V, FOURS>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((balance_kernel<L, LANES, V, FOURS>), grid, block, (256 * V + a.experts) * 4, s, a);
    HIP_TRY(hipGetLastError());
    return FICCO_OK;
}
template <class L>
int launch(const BalanceLaunch &a, bool backward, hipStream_t s)
{
    // whole fours of logits where a lane has four or more (not by where the rows lie: equal calls give equal bits)
    const bool fours = a.experts % 4 == 0;
    if (a.experts <= 8) return launch_t<L, 8, 1, false>(a, backward, s);
    if (a.experts <= 16) return launch_t<L, 16, 1, false>(a, backward, s);
    if (a.experts <= 32) return launch_t<L, 32, 1, false>(a, backward, s);
    if (a.experts <= 64) return launch_t<L, 64, 1, false>(a, backward, s);
    if (a.experts <= 128) return launch_t<L, 64, 2, false>(a, backward, s);
    if (a.experts <= 256) return fours ? launch_t<L, 64, 4, true>(a, backward, s) : launch_t<L, 64, 4, false>(a, backward, s);
    if (a.experts <= 512) return fours ? launch_t<L, 64, 8, true>(a, backward, s) : launch_t<L, 64, 8, false>(a, backward, s);
    return fours ? launch_t<L, 64, 16, true>(a, backward, s) : launch_t<L, 64, 16, false>(a, backward, s);
}

int forward(const ficco_expert_balance_t *op, const void *logits, const void *ids, const void *valid, void *counts, void *group_valid, void *loss,
            void *workspace, int64_t workspace_bytes, hipStream_t s)
{
    ficco_expert_balance_t o;
    int rc = checked(op, &o);
    if (rc) return rc;
    const bool none = o.tokens == 0;
    rc = check_args({{logits, o.logits_type == FICCO_F32 ? 4 : 2, none || !loss}, {ids, 4, none}, {valid, 1, true}, {counts, 4, none}, {group_valid, 4, none},
                     {loss, 4, true}, {workspace, 16, true}});
    if (rc) return rc;
    if (none) {
        if (!loss) return FICCO_OK;
        hipLaunchKernelGGL(balance_loss_kernel, dim3(1), dim3(1024), 0, s, nullptr, 0, (float *)loss);
        HIP_TRY(hipGetLastError());
        return FICCO_OK;
    }
    const Chunks c = forward_chunks(o);
    const Workspace w = workspace_of(o);
    if (w.bytes > 0 && (!workspace || workspace_bytes < w.bytes)) return FICCO_ERR_ARG;
    unsigned char *const ws = (unsigned char *)workspace;
    BalanceLaunch a = launch_of(o, c);
    a.logits = logits;
    a.ids = (const int32_t *)ids;
    a.valid = (const uint8_t *)valid;
    a.counts = (int32_t *)counts;
    a.group_valid = (int32_t *)group_valid;
    a.loss = (float *)loss;
    a.part_p = (float *)(ws + w.p);
    a.part_c = (int32_t *)(ws + w.c);
    a.part_n = (int32_t *)(ws + w.n);
    a.terms = (float *)(ws + w.terms);
    a.n_terms = (int32_t)w.n_terms;
    rc = o.logits_type == FICCO_F32 ? launch<float>(a, false, s) : launch<uint16_t>(a, false, s);
    if (rc) return rc;
    if (c.per_group > 1) {
        hipLaunchKernelGGL(balance_group_kernel, dim3((unsigned)c.groups, (unsigned)c.joins), dim3(1024), 0, s, a);
        HIP_TRY(hipGetLastError());
    }
    if (loss && w.n_terms > 1) {
        hipLaunchKernelGGL(balance_loss_kernel, dim3(1), dim3(1024), 0, s, a.terms, a.n_terms, (float *)loss);
        HIP_TRY(hipGetLastError());
    }
    return FICCO_OK;
}

int backward(const ficco_expert_balance_t *op, const void *logits, const void *valid, const void *counts, const void *group_valid, const void *dloss,
             void *dlogits, hipStream_t s)
{
    ficco_expert_balance_t o;
    int rc = checked(op, &o);
    if (rc) return rc;
    const bool none = o.tokens == 0;
    const int align = o.logits_type == FICCO_F32 ? 4 : 2;
    rc = check_args({{logits, align, none}, {valid, 1, true}, {counts, 4, none}, {group_valid, 4, none}, {dloss, 4, true}, {dlogits, align, none}});
    if (rc || none) return rc;
    BalanceLaunch a = launch_of(o, backward_chunks(o));
    a.logits = logits;
    a.valid = (const uint8_t *)valid;
    a.counts = (int32_t *)const_cast<void *>(counts);
    a.group_valid = (int32_t *)const_cast<void *>(group_valid);
    a.dloss = (const float *)dloss;
    a.dlogits = dlogits;
    return o.logits_type == FICCO_F32 ? launch<float>(a, true, s) : launch<uint16_t>(a, true, s);
}

}  // namespace
}  // namespace ficco

using namespace ficco;

extern "C" {

int ficco_expert_balance_workspace(const ficco_expert_balance_t *op, int64_t *bytes)
{
    return guarded([&] {
        ficco_expert_balance_t o;
        if (!bytes) return (int)FICCO_ERR_ARG;
        const int rc = checked(op, &o);
        if (rc) return rc;
        *bytes = o.tokens ? workspace_of(o).bytes : 0;
        return (int)FICCO_OK;
    });
}

int ficco_expert_balance(const ficco_expert_balance_t *op, const void *logits, const void *ids, const void *valid, void *counts, void *group_valid,
                         void *loss, void *workspace, int64_t workspace_bytes, void *stream)
{
    return guarded([&] { return forward(op, logits, ids, valid, counts, group_valid, loss, workspace, workspace_bytes, (hipStream_t)stream); });
}

int ficco_expert_balance_backward(const ficco_expert_balance_t *op, const void *logits, const void *valid, const void *counts, const void *group_valid,
                                  const void *dloss, void *dlogits, void *stream)
{
    return guarded([&] { return backward(op, logits, valid, counts, group_valid, dloss, dlogits, (hipStream_t)stream); });
}

}  // extern "C"

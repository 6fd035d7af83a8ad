// The whole layer for a few tokens, in two launches.
//
//   few_logits   router logits, each as eight partial sums; clears the counters of the second launch
//   few_ffn      top-K, expert lists, both products of the experts that got a row, the weighted sum
//
// The layer is bound by reading the touched experts' weights once; everything else is latency.  few_ffn is a persistent grid
// whose workgroups draw their work from one counter, in this order:
//   tokens   (more than kRouteAll tokens) top-K of eight tokens, one per wavefront; up to kRouteAll tokens every workgroup
//            selects for itself, which is quicker than waiting for another's answer
//   gate/up  (expert, 16 columns of F): both products of the expert's rows, the activation into the workspace
//   down     16 or 32 columns of H over ALL touched experts: a token's sum over its K experts is made in one workgroup, in
//            ascending order of experts, so there is no third exchange and equal calls give equal bits
// A draw waits for all draws of the kind before it to be finished.  Whoever holds one of those runs and waits for nothing
// later, so every wait ends, however few workgroups of the grid are resident (several calls on several streams included).
// The activation goes from XCD to XCD: it is written through, counted when the stores are acknowledged, and read after the
// caches have been told to drop what they hold.
//
// Rows of an expert are the set bits of a mask of 64 tokens: slot and count are population counts, in ascending n.
#include <math.h>

#include "common.h"
#include "few.h"
#include "few_stream.h"
#include "select.h"

namespace moe {

constexpr int kFewWaves = 8, kFewThreads = kFewWaves * kWave;
constexpr int kParts = 8; // partial sums of a logit between the launches
constexpr int kRouteAll = 16;
constexpr int kMaxRows = MOE_FEW_TOKENS * MOE_MAX_TOPK;
constexpr int kWaitPolls = 1 << 24; // seconds: never reached (see above), so that nothing can hang all the same

struct FewCounters { // a cache line each
    uint32_t drawn, pad0[31];
    uint32_t routed, pad1[31];
    uint32_t activated, pad2[31];
};

// ------------------------------------------------------------------------
// Logits in moe_route's order (route.hip, "R64"): partial l of 64 takes h = l, l + 64, ... by single fused multiply-adds,
// which v_mfma_f32_16x16x1_4B_f32 does for four partials of 16 tokens x 16 experts at a time; then rounds 32, 16, ... 1.
// A workgroup has sixteen experts and the eight partials l = j, j + 8, ... (wavefront 0: the first four), which rounds 32,
// 16 and 8 make one; the reader does rounds 4, 2, 1.  So even one token's router runs on E / 2 workgroups, and an XCD
// (j = blockIdx.x % 8) has rows of W_r of its own.  Latency bound: all loads of 64 steps are in flight at once.
// ------------------------------------------------------------------------
template <bool kBf16>
__global__ __launch_bounds__(2 * kWave) void few_logits(const void *__restrict__ x, int N, int H, const float *__restrict__ W_r,
                                                        int E, float *__restrict__ parts, FewCounters *counters)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kBatch = 32;
    __shared__ float fold[16 * kWave];
    const int lane = threadIdx.x % kWave, c = lane % 16, blk = lane / 16;
    const int half = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int j = (int)blockIdx.x % kParts, e0 = (int)blockIdx.x / kParts * 16, n0 = (int)blockIdx.y * 16;
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0)
        counters->drawn = counters->routed = counters->activated = 0;
    const int l = j + 8 * (4 * half + blk);
    const int tok = n0 + c < N ? n0 + c : N - 1, e = e0 + c < E ? e0 + c : E - 1;
    const int steps = (H + kWave - 1) / kWave;
    struct Batch {
        uint32_t x[kBatch];
        float w[kBatch];
    };
    auto fetch = [&](Batch &b, int s0) {
#pragma unroll
        for (int s = 0; s < kBatch; ++s) {
            const int h = (s0 + s) * kWave + l;
            const bool in = h < H; // (past the end: zeros)
            const float w = W_r[(int64_t)(in ? h : 0) * E + e];
            b.w[s] = in ? w : 0.0f;
            if constexpr (kBf16) {
                const uint32_t v = static_cast<const uint16_t *>(x)[(int64_t)tok * H + (in ? h : 0)];
                b.x[s] = in ? v << 16 : 0u;
            } else {
                const uint32_t v = static_cast<const uint32_t *>(x)[(int64_t)tok * H + (in ? h : 0)];
                b.x[s] = in ? v : 0u;
            }
        }
    };
    f32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r)
        acc[r] = 0.0f;
    auto multiply = [&](const Batch &b) {
#pragma unroll
        for (int s = 0; s < kBatch; ++s)
            acc = __builtin_amdgcn_mfma_f32_16x16x1f32(__uint_as_float(b.x[s]), b.w[s], acc, 0, 0, 0);
    };
    Batch b0, b1;
    fetch(b0, 0);
    for (int s = 0; s < steps; s += 2 * kBatch) {
        fetch(b1, s + kBatch);
        multiply(b0);
        if (s + 2 * kBatch < steps)
            fetch(b0, s + 2 * kBatch);
        multiply(b1);
    }
    // register 4 b + t of lane (q, c): partial of block b, token 4 q + t, expert c
    if (half == 1)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            fold[r * kWave + lane] = acc[r];
    __syncthreads();
    if (half == 1 || e0 + c >= E)
        return;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        float v[4];
#pragma unroll
        for (int b = 0; b < 4; ++b)
            v[b] = acc[4 * b + t] + fold[(4 * b + t) * kWave + lane];
        const int n = n0 + 4 * blk + t;
        if (n < N)
            parts[((int64_t)n * kParts + j) * E + e0 + c] = (v[0] + v[2]) + (v[1] + v[3]);
    }
#endif
}

// ------------------------------------------------------------------------
struct FewKernelArgs {
    FewArgs l;
    const float *parts;
    FewCounters *counters;
};

#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ float silu_mul_f32(float g, float u) { return g / (1.0f + expf(-g)) * u; }

// Thread 0 only: waits until *count is `want`.
__device__ __forceinline__ bool few_wait(const uint32_t *count, uint32_t want)
{
    for (int i = 0; i < kWaitPolls; ++i) {
        if (__hip_atomic_load(count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == want)
            return true;
        __builtin_amdgcn_s_sleep(1);
    }
    return false;
}

__device__ __forceinline__ Pick few_select(const FewKernelArgs &g, int n)
{
    const FewArgs &l = g.l;
    const float *const parts = g.parts + (int64_t)n * kParts * l.E;
    auto logit_of = [&](int e) {
        float p[kParts];
#pragma unroll
        for (int j = 0; j < kParts; ++j)
            p[j] = parts[j * l.E + e];
#pragma unroll
        for (int s = kParts / 2; s >= 1; s >>= 1)
#pragma unroll
            for (int j = 0; j < s; ++j)
                p[j] = p[j] + p[j + s];
        return l.bias ? p[0] + l.bias[e] : p[0];
    };
    return l.E <= kWave       ? select_top<1>(logit_of, l.E, l.K, l.score_mode)
           : l.E <= 2 * kWave ? select_top<2>(logit_of, l.E, l.K, l.score_mode)
           : l.E <= 4 * kWave ? select_top<4>(logit_of, l.E, l.K, l.score_mode)
                              : select_top<MOE_MAX_EXPERTS / kWave>(logit_of, l.E, l.K, l.score_mode);
}

// The experts that got a row, in ascending order, and their rows: slots [offset[a], offset[a + 1]).
struct FewLists {
    int active;
    uint16_t expert[MOE_MAX_EXPERTS], offset[MOE_MAX_EXPERTS + 1];
    uint8_t token[kMaxRows];
    float weight[kMaxRows];
};
struct FewRouting { // while the lists are made
    uint64_t mask[MOE_MAX_EXPERTS];  // of tokens
    uint16_t first[MOE_MAX_EXPERTS]; // slot
    uint16_t pick[kMaxRows];
    float weight[kMaxRows];
    uint32_t wave_sum[kFewWaves];
};

// All threads; r.pick and r.weight are there, r.mask is zero.
__device__ __forceinline__ void few_make_lists(FewLists &lists, FewRouting &r, int N, int K, int E)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    for (int at = threadIdx.x; at < N * K; at += kFewThreads)
        atomicOr(reinterpret_cast<unsigned long long *>(&r.mask[r.pick[at]]), 1ull << (at / K));
    __syncthreads();
    // two experts per thread; rows in the low half, experts with a row in the high one
    constexpr int kPer = MOE_MAX_EXPERTS / kFewThreads;
    uint32_t mine[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = threadIdx.x * kPer + i;
        const uint32_t rows = e < E ? (uint32_t)__popcll(r.mask[e]) : 0u;
        mine[i] = rows | (rows ? 1u << 16 : 0u);
        sum += mine[i];
    }
    uint32_t up_to = sum;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        const uint32_t v = __shfl_up(up_to, s);
        up_to += lane >= s ? v : 0u;
    }
    if (lane == kWave - 1)
        r.wave_sum[wave] = up_to;
    __syncthreads();
    uint32_t at = up_to - sum, all = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        at += w < wave ? r.wave_sum[w] : 0u;
        all += r.wave_sum[w];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (mine[i]) {
            const int e = threadIdx.x * kPer + i;
            lists.expert[at >> 16] = (uint16_t)e;
            lists.offset[at >> 16] = r.first[e] = (uint16_t)at;
        }
        at += mine[i];
    }
    if (threadIdx.x == 0) {
        lists.active = (int)(all >> 16);
        lists.offset[all >> 16] = (uint16_t)all;
    }
    __syncthreads();
    for (int p = threadIdx.x; p < N * K; p += kFewThreads) {
        const int e = r.pick[p], n = p / K;
        const int slot = r.first[e] + (int)__popcll(r.mask[e] & ((1ull << n) - 1));
        lists.token[slot] = (uint8_t)n;
        lists.weight[slot] = r.weight[p];
    }
    __syncthreads();
}

// Lines in flight per wavefront: what the registers of a wavefront hold (128 with kMaxTT == 1: two workgroups on a compute
// unit, else 256).
template <int kForm, int kTT, int kMaxTT>
constexpr int few_depth()
{
    if (kMaxTT == 1)
        return kTT ? 3 : 4;
    return kTT <= 1 ? 5 : kTT == 2 ? 3 : 2;
}

// One tile of the gate/up projection: columns [f0, f0 + 16) for slots [s0, s0 + rows) of an expert.
template <int kForm, int kTT, int kMaxTT>
__device__ __forceinline__ void few_gate_up_tile(const FewArgs &l, const FewLists &lists, float *red, int expert, int s0, int rows, int f0)
{
    using Form = FewForm<kForm>;
    constexpr int kValues = kFewValues<kForm, kTT>;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t row = (int64_t)expert * l.F + f0, end = (int64_t)(expert + 1) * l.F;
    const Panel panels[2] = {panel_of<kForm>(l.gate, row, end, l.H, l.scale_cols_h), panel_of<kForm>(l.up, row, end, l.H, l.scale_cols_h)};
    const uint32_t x_row = (uint32_t)l.H * Form::kElt;
    const auto act = act_rows(l.x, (uint32_t)l.N * x_row, rows, [&](int r) { return lists.token[s0 + r] * x_row; });
    const int lines = (l.H + Form::kLineCols - 1) / Form::kLineCols, share = (lines + kFewWaves - 1) / kFewWaves;
    const int first = wave * share, last = first + share < lines ? first + share : lines;
    FewSums<kForm, kTT, 2> sums;
    sums.clear();
    few_stream<kForm, kTT, 2, few_depth<kForm, kTT, kMaxTT>()>(sums, panels, act, {l.H, l.scale_cols_h, l.group}, first, last);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int v = 0; v < kValues; ++v)
            red[((wave * 2 + c) * kValues + v) * kWave + lane] = sums.value(c, v);
    few_barrier();
    for (int v = wave; v < kValues; v += kFewWaves) {
        float total[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            total[c] = red[(c * kValues + v) * kWave + lane];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w)
                total[c] += red[((w * 2 + c) * kValues + v) * kWave + lane];
        }
        const float a = silu_mul_f32(total[0], total[1]);
        const int r = few_row_of<kForm, kTT>(v), f = f0 + lane % 16;
        const bool there = r < rows && f < l.F;
        const int64_t at = (int64_t)(s0 + r) * l.F + f;
        if constexpr (kForm == kFewF32) {
            if (there)
                __hip_atomic_store(static_cast<uint32_t *>(l.a) + at, __float_as_uint(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        } else { // the even lane stores both columns (F is even)
            const uint32_t both = pack_bf16x2(a, __shfl_xor(a, 1));
            if (there && lane % 2 == 0)
                __hip_atomic_store(reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(l.a) + at), both, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
        }
    }
}

// Lines [first, last) of an expert's part of the down projection for columns [h0, h0 + 16 kCT): the weighted rows are added
// to the wavefront's own sums per token.
template <int kForm, int kTT, int kCT, int kMaxTT>
__device__ __forceinline__ void few_down_part(const FewArgs &l, const FewLists &lists, float *token_sums, int expert, int s0, int rows,
                                              int h0, int first, int last)
{
    using Form = FewForm<kForm>;
    const int64_t row = (int64_t)expert * l.H + h0, end = (int64_t)(expert + 1) * l.H;
    Panel panels[kCT];
#pragma unroll
    for (int c = 0; c < kCT; ++c)
        panels[c] = panel_of<kForm>(l.down, row + 16 * c, end, l.F, l.scale_cols_f);
    const uint32_t a_row = (uint32_t)l.F * Form::kElt;
    const auto act = act_rows(static_cast<const unsigned char *>(l.a) + (int64_t)s0 * a_row, (uint32_t)rows * a_row, rows,
                              [&](int r) { return r * a_row; });
    FewSums<kForm, kTT, kCT> sums;
    sums.clear();
    few_stream<kForm, kTT, kCT, few_depth<kForm, kTT, kMaxTT>()>(sums, panels, act, {l.F, l.scale_cols_f, l.group}, first, last);
#pragma unroll
    for (int v = 0; v < kFewValues<kForm, kTT>; ++v) {
        const int r = few_row_of<kForm, kTT>(v);
        if (r < rows) { // (a token has an expert once: the lanes of a wavefront meet nowhere)
            const float w = lists.weight[s0 + r];
            float *const at = token_sums + lists.token[s0 + r] * (16 * kCT) + threadIdx.x % 16;
#pragma unroll
            for (int c = 0; c < kCT; ++c)
                at[16 * c] += w * sums.value(c, v);
        }
    }
}

// Calls f with the smallest form that holds `rows`.
template <int kForm, int kMaxTT, class F>
__device__ __forceinline__ void few_by_rows(int rows, F f)
{
    if (rows <= FewForm<kForm>::kFewRows)
        f(std::integral_constant<int, 0>{});
    else if (kMaxTT == 1 || rows <= 16)
        f(std::integral_constant<int, 1>{});
    else if (kMaxTT == 2 || rows <= 32)
        f(std::integral_constant<int, (kMaxTT < 2 ? 1 : 2)>{});
    else
        f(std::integral_constant<int, kMaxTT>{});
}
#endif

// kMaxTT: sixteens of rows that an expert can have (N).  kCT: sixteens of columns of a down tile.
template <int kForm, int kMaxTT, int kCT>
__global__ __launch_bounds__(kFewThreads, kMaxTT == 1 ? 4 : 2) void few_ffn(FewKernelArgs g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using Form = FewForm<kForm>;
    constexpr int kRed = kFewWaves * 2 * (kMaxTT > 1 ? 4 * kMaxTT : 4) * kWave, kSums = kFewWaves * 16 * kMaxTT * 16 * kCT;
    __shared__ union {
        FewRouting routing;
        float red[kRed];
        float sums[kSums];
    } sh;
    __shared__ FewLists lists;
    __shared__ uint32_t box; // the draw
    __shared__ bool failed;
    const FewArgs &l = g.l;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    auto draw = [&]() { return __hip_atomic_fetch_add(&g.counters->drawn, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    uint32_t next = 0; // thread 0's
    if (threadIdx.x == 0) {
        next = draw();
        failed = false;
    }
    for (int e = threadIdx.x; e < l.E; e += kFewThreads)
        sh.routing.mask[e] = 0;
    uint32_t token_draws = 0;
    if (l.N <= kRouteAll) {
        for (int n = wave; n < l.N; n += kFewWaves) {
            const Pick p = few_select(g, n);
            if (lane < l.K) {
                sh.routing.pick[n * l.K + lane] = (uint16_t)p.expert;
                sh.routing.weight[n * l.K + lane] = p.weight;
                if (blockIdx.x == 0) {
                    l.topk_idx[n * l.K + lane] = p.expert;
                    l.topk_w[n * l.K + lane] = p.weight;
                }
            }
        }
    } else {
        token_draws = (uint32_t)(l.N + kFewWaves - 1) / kFewWaves;
        for (;;) {
            if (threadIdx.x == 0)
                box = next;
            __syncthreads();
            const uint32_t t = box;
            if (t >= token_draws)
                break;
            if (threadIdx.x == 0)
                next = draw();
            const int n = (int)t * kFewWaves + wave;
            if (n < l.N) {
                const Pick p = few_select(g, n);
                if (lane < l.K) {
                    __hip_atomic_store(l.topk_idx + n * l.K + lane, p.expert, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    __hip_atomic_store(l.topk_w + n * l.K + lane, p.weight, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (threadIdx.x == 0)
                __hip_atomic_fetch_add(&g.counters->routed, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        if (threadIdx.x == 0 && !few_wait(&g.counters->routed, token_draws))
            failed = true;
        __syncthreads();
        for (int p = threadIdx.x; p < l.N * l.K; p += kFewThreads) {
            const int e = __hip_atomic_load(l.topk_idx + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            sh.routing.pick[p] = (uint16_t)((unsigned)e < (unsigned)l.E ? e : 0);
            sh.routing.weight[p] = __hip_atomic_load(l.topk_w + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    __syncthreads();
    few_make_lists(lists, sh.routing, l.N, l.K, l.E);

    // ---- gate/up tiles
    const int f_tiles = (l.F + 15) / 16;
    const uint32_t gate_up = (uint32_t)(lists.active * f_tiles);
    uint32_t item;
    for (;;) {
        if (threadIdx.x == 0)
            box = next;
        __syncthreads(); // (the reads of red are done)
        item = box - token_draws;
        if (item >= gate_up)
            break;
        if (threadIdx.x == 0)
            next = draw();
        const int at = __builtin_amdgcn_readfirstlane((int)item / f_tiles), f0 = __builtin_amdgcn_readfirstlane((int)item % f_tiles) * 16;
        const int expert = __builtin_amdgcn_readfirstlane(lists.expert[at]), s0 = __builtin_amdgcn_readfirstlane(lists.offset[at]);
        const int rows = __builtin_amdgcn_readfirstlane(lists.offset[at + 1]) - s0;
        few_by_rows<kForm, kMaxTT>(rows, [&](auto tt) {
            few_gate_up_tile<kForm, decltype(tt)::value, kMaxTT>(l, lists, sh.red, expert, s0, rows, f0);
        });
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // my part of the activation is in memory
        __syncthreads();
        if (threadIdx.x == 0)
            __hip_atomic_fetch_add(&g.counters->activated, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }

    // ---- down tiles
    const uint32_t down = (uint32_t)((l.H + 16 * kCT - 1) / (16 * kCT));
    item -= gate_up;
    if (item >= down)
        return;
    if (threadIdx.x == 0 && !few_wait(&g.counters->activated, gate_up))
        failed = true;
    __syncthreads();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    const int lines = (l.F + Form::kLineCols - 1) / Form::kLineCols, all = lines * lists.active;
    const int from = (int)((int64_t)all * wave / kFewWaves), to = (int)((int64_t)all * (wave + 1) / kFewWaves);
    const int tile = l.N * 16 * kCT;
    for (;;) {
        if (threadIdx.x == 0)
            next = draw();
        const int h0 = (int)item * 16 * kCT;
        float *const mine = sh.sums + wave * tile;
        for (int p = lane; p < tile; p += kWave)
            mine[p] = 0.0f;
        for (int line = from; line < to;) {
            const int at = line / lines, first = line - at * lines, last = to - at * lines < lines ? to - at * lines : lines;
            const int expert = __builtin_amdgcn_readfirstlane(lists.expert[at]), s0 = __builtin_amdgcn_readfirstlane(lists.offset[at]);
            const int rows = __builtin_amdgcn_readfirstlane(lists.offset[at + 1]) - s0;
            few_by_rows<kForm, kMaxTT>(rows, [&](auto tt) {
                few_down_part<kForm, decltype(tt)::value, kCT, kMaxTT>(l, lists, mine, expert, s0, rows, h0, first, last);
            });
            line += last - first;
        }
        __syncthreads();
        for (int p = threadIdx.x * 2; p < tile; p += kFewThreads * 2) { // (H and F are even)
            float v[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                v[u] = sh.sums[p + u];
#pragma unroll
                for (int w = 1; w < kFewWaves; ++w)
                    v[u] += sh.sums[w * tile + p + u];
                if (failed)
                    v[u] = NAN;
            }
            const int n = p / (16 * kCT), h = h0 + p % (16 * kCT);
            if (h < l.H) {
                if constexpr (kForm == kFewF32)
                    *reinterpret_cast<f32x2 *>(static_cast<float *>(l.out) + (int64_t)n * l.H + h) = f32x2{v[0], v[1]};
                else
                    *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(l.out) + (int64_t)n * l.H + h) = pack_bf16x2(v[0], v[1]);
            }
        }
        if (threadIdx.x == 0)
            box = next;
        __syncthreads();
        item = box - token_draws - gate_up;
        if (item >= down)
            break;
    }
#endif
}

struct FewWorkspace {
    FewCounters *counters;
    float *parts;
    void *a;
    size_t bytes;
};

static FewWorkspace few_carve(void *ws, int64_t N, int E, int K, int64_t F, int dtype)
{
    unsigned char *const w = static_cast<unsigned char *>(ws);
    const size_t parts = sizeof(FewCounters), a = parts + ((size_t)N * kParts * E * sizeof(float) + 127) / 128 * 128;
    return {reinterpret_cast<FewCounters *>(w), reinterpret_cast<float *>(w + parts), w + a,
            a + ((size_t)N * K * F * (dtype == MOE_BF16 ? 2 : 4) + 127) / 128 * 128};
}

size_t few_workspace_bytes(int64_t N, int64_t H, int E, int K, int64_t F, int dtype)
{
    (void)H;
    return few_carve(nullptr, N, E, K, F, dtype).bytes;
}

template <int kForm>
static void launch_ffn(const FewKernelArgs &g, hipStream_t st)
{
    const int cus = compute_units();
    const bool wide = g.l.N * g.l.K > 4 * g.l.E;
    const dim3 block(kFewThreads);
    if (g.l.N <= 16) {
        if (wide)
            hipLaunchKernelGGL((few_ffn<kForm, 1, 2>), dim3(2 * cus), block, 0, st, g);
        else
            hipLaunchKernelGGL((few_ffn<kForm, 1, 1>), dim3(2 * cus), block, 0, st, g);
    } else {
        if (wide)
            hipLaunchKernelGGL((few_ffn<kForm, 4, 2>), dim3(cus), block, 0, st, g);
        else
            hipLaunchKernelGGL((few_ffn<kForm, 4, 1>), dim3(cus), block, 0, st, g);
    }
}

int launch_layer_few(const FewArgs &args, int dtype, int format, hipStream_t st)
{
    const FewWorkspace w = few_carve(args.ws, args.N, args.E, args.K, args.F, dtype);
    FewKernelArgs g = {args, w.parts, w.counters};
    g.l.a = w.a;
    const dim3 grid((unsigned)(ceil_div(args.E, 16) * kParts), (unsigned)ceil_div(args.N, 16));
    if (dtype == MOE_BF16)
        hipLaunchKernelGGL(few_logits<true>, grid, dim3(2 * kWave), 0, st, args.x, args.N, args.H, args.W_r, args.E, w.parts, w.counters);
    else
        hipLaunchKernelGGL(few_logits<false>, grid, dim3(2 * kWave), 0, st, args.x, args.N, args.H, args.W_r, args.E, w.parts, w.counters);
    if (format == MOE_Q4_FP4)
        launch_ffn<kFewFp4>(g, st);
    else if (format == MOE_Q4_INT4)
        launch_ffn<kFewInt4>(g, st);
    else if (dtype == MOE_BF16)
        launch_ffn<kFewBf16>(g, st);
    else
        launch_ffn<kFewF32>(g, st);
    return check_launch("moe_layer_few");
}

}  // namespace moe

// The whole layer for a few tokens, in two launches.
//
//   few_logits   router logits, each as eight partial sums; clears the flags of the second launch
//   few_ffn      top-K, expert lists, both products of the experts that got a row, the weighted sum
//
// The layer is bound by reading the touched experts' weights once; everything else is latency.  few_ffn has one workgroup
// per compute unit, with a fixed share of each step:
//   tokens   (more than kRouteAll) top-K of eight tokens, one per wavefront; up to kRouteAll tokens every workgroup selects
//            for itself, which is quicker than waiting for another's answer
//   gate/up  items (expert, 16 columns of F): both products of the expert's rows and the activation, into the workspace.
//            The wavefronts share the reduction; a wavefront's stream of weights runs on from item to item
//   down     a few columns of H over ALL touched experts (as many as make a share for every workgroup): a token's sum over
//            its K experts is made in one workgroup, so there is no third exchange and equal calls give equal bits
// Shares are fixed because drawing them costs more than it gives: atomics on one address are served one in 12 ns (512
// workgroups that drew from one counter and polled another: one token 64 us instead of 20).
//
// What a step needs from other workgroups is said by a flag per share.  A workgroup that has waited for longer than any share
// takes does the missing share itself (a second time, with the same bits, if its owner is only late): every wait ends, however
// few workgroups of the grid are resident, several calls on several streams included.
// The activation goes from XCD to XCD.  It is written through and a share's flag is set once its stores are acknowledged.  It
// is read by ordinary loads: a cache line belongs to one item, so no XCD can hold one that was read or written in part before
// its item was complete.  (Telling the caches to drop what they hold takes 5 - 9 us.)
//
// Rows of an expert are the set bits of a mask of 64 tokens: slot and count are population counts, in ascending n.  Experts are
// taken in four classes by their rows (few_stream.h's forms), each a stream of its own.
#pragma once

#include <math.h>

#include "common.h"
#include "few.h"
#include "few_stream.h"
#include "select.h"

namespace moe {

constexpr int kFewWaves = 8, kFewThreads = kFewWaves * kWave;
constexpr int kParts = 8; // partial sums of a logit between the launches
constexpr int kRouteAll = 8;
constexpr int kMaxRows = MOE_FEW_TOKENS * MOE_MAX_TOPK;
constexpr int kTokenFlags = MOE_FEW_TOKENS / kFewWaves, kMaxShares = 1024, kFlags = 32 + kMaxShares; // tokens', then shares'
constexpr int kDefaultPatience = 1 << 15; // polls (about a microsecond each): longer than a share takes

// An expert's rows of the activation are a multiple of this many, so that an item of 16 columns is whole cache lines.
template <int kForm>
constexpr int kRowPad = 128 / (16 * FewForm<kForm>::kElt);
constexpr int kMaxSlots = kMaxRows + 3 * MOE_MAX_EXPERTS;

// ------------------------------------------------------------------------
struct FewKernelArgs {
    FewArgs l;
    const float *parts;
    uint32_t *flags;
    int shares;    // of gate/up items
    int down_cols; // columns of H of a down tile, at most 16 kCT
    int patience;
};

#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ float silu_mul_f32(float g, float u) { return g / (1.0f + expf(-g)) * u; }

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

// The experts that got a row, by class and in ascending order within it, and their rows: slots from base on.
struct FewLists {
    int begin[5]; // of the classes: at most kFewRows rows, 16, 32, 64
    uint16_t expert[MOE_MAX_EXPERTS], base[MOE_MAX_EXPERTS];
    uint8_t rows[MOE_MAX_EXPERTS];
    uint8_t token[kMaxSlots];
    float weight[kMaxSlots];
};
struct FewRouting { // while the lists are made
    uint64_t mask[MOE_MAX_EXPERTS];  // of tokens
    uint16_t first[MOE_MAX_EXPERTS]; // slot
    uint16_t pick[kMaxRows];
    float weight[kMaxRows];
    uint64_t wave_sum[kFewWaves];
};

// All threads; r.pick and r.weight are there, r.mask is zero.
template <int kForm>
__device__ __forceinline__ void few_make_lists(FewLists &lists, FewRouting &r, int N, int K, int E)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    for (int at = threadIdx.x; at < N * K; at += kFewThreads)
        atomicOr(reinterpret_cast<unsigned long long *>(&r.mask[r.pick[at]]), 1ull << (at / K));
    __syncthreads();
    // Two experts per thread.  Sums: slots in the low 13 bits, then experts of each class in 11 bits.
    constexpr int kPer = MOE_MAX_EXPERTS / kFewThreads;
    auto shift_of = [](int rows) { return 13 + 11 * (rows <= FewForm<kForm>::kFewRows ? 0 : rows <= 16 ? 1 : rows <= 32 ? 2 : 3); };
    uint64_t mine[kPer], sum = 0;
    int rows[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = threadIdx.x * kPer + i;
        rows[i] = e < E ? (int)__popcll(r.mask[e]) : 0;
        mine[i] = rows[i] ? (uint64_t)((rows[i] + kRowPad<kForm> - 1) / kRowPad<kForm> * kRowPad<kForm>) | 1ull << shift_of(rows[i]) : 0;
        sum += mine[i];
    }
    uint64_t up_to = sum;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        const uint64_t v = __shfl_up((unsigned long long)up_to, s);
        up_to += lane >= s ? v : 0;
    }
    if (lane == kWave - 1)
        r.wave_sum[wave] = up_to;
    __syncthreads();
    uint64_t at = up_to - sum, all = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        at += w < wave ? r.wave_sum[w] : 0;
        all += r.wave_sum[w];
    }
    int begin[5] = {0, 0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < 4; ++c)
        begin[c + 1] = begin[c] + (int)(all >> (13 + 11 * c) & 0x7FF);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (rows[i]) {
            const int e = threadIdx.x * kPer + i, shift = shift_of(rows[i]);
            const int place = begin[(shift - 13) / 11] + (int)(at >> shift & 0x7FF);
            lists.expert[place] = (uint16_t)e;
            lists.rows[place] = (uint8_t)rows[i];
            lists.base[place] = r.first[e] = (uint16_t)(at & 0x1FFF);
        }
        at += mine[i];
    }
    if (threadIdx.x == 0)
#pragma unroll
        for (int c = 0; c < 5; ++c)
            lists.begin[c] = begin[c];
    __syncthreads();
    for (int p = threadIdx.x; p < N * K; p += kFewThreads) {
        const int e = r.pick[p], n = p / K;
        const int slot = r.first[e] + (int)__popcll(r.mask[e] & ((1ull << n) - 1));
        lists.token[slot] = (uint8_t)n;
        lists.weight[slot] = r.weight[p];
    }
    __syncthreads();
}

// All threads: -1 once all flags are set, or one that still is not after `patience` polls.
__device__ __forceinline__ int few_missing(const uint32_t *flags, int count, int patience, int *box)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    for (int poll = 0;; ++poll) {
        int miss = 0x7FFFFFFF;
        for (int i = threadIdx.x; i < count; i += kFewThreads)
            if (__hip_atomic_load(flags + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0)
                miss = miss < i ? miss : i;
        const uint64_t m = __ballot(miss != 0x7FFFFFFF);
        const int mine = m ? __builtin_amdgcn_readlane(miss, __builtin_ctzll(m)) : 0x7FFFFFFF;
        if (lane == 0)
            box[wave] = mine;
        few_barrier();
        int first = 0x7FFFFFFF;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w)
            first = first < box[w] ? first : box[w];
        first = __builtin_amdgcn_readfirstlane(first);
        few_barrier();
        if (first == 0x7FFFFFFF)
            return -1;
        if (poll >= patience)
            return first;
        __builtin_amdgcn_s_sleep(4);
    }
}

// All threads: what this workgroup has stored is in memory; then the flag says so.
__device__ __forceinline__ void few_signal(uint32_t *flag)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    few_barrier();
    if (threadIdx.x == 0)
        __hip_atomic_store(flag, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Lines in flight per wavefront: what 256 registers hold beside a line's products (registers of a line in the comment).
template <int kForm, int kTT, int kCT>
constexpr int few_depth()
{
    if (kForm == kFewInt4)
        return kTT == 0 ? 6 : kTT == 1 ? 4 : 2;
    if (FewForm<kForm>::kQ4) // 5 kCT + 4, 16, 32, 64
        return kTT == 0 ? 8 : kTT == 1 ? 6 : kTT == 2 ? 4 : 2;
    return kTT <= 1 ? (kCT == 1 ? 8 : 6) : kTT == 2 ? 4 : 3; // 8 kCT + 4, 8, 16, 32
}

// Where the activation of `rows` rows from slot `base` on is: sixteen columns of all (padded) rows side by side.
template <int kForm>
__device__ __forceinline__ FewActs few_activation(const FewArgs &l, int base, int rows)
{
    constexpr int kElt = FewForm<kForm>::kElt;
    const int padded = (rows + kRowPad<kForm> - 1) / kRowPad<kForm> * kRowPad<kForm>, cols = (l.F + 15) / 16 * 16;
    return {static_cast<const unsigned char *>(l.a) + (int64_t)base * cols * kElt, (uint32_t)padded * (uint32_t)cols * kElt,
            (uint32_t)padded * 16 * kElt, rows};
}

// Gate/up items of one class: (expert, 16 columns of F), every `step`-th; the eight wavefronts share the reduction.
template <int kForm, int kTT>
struct GateUp {
    using Form = FewForm<kForm>;
    const FewArgs &l;
    const FewLists &lists;
    float *red; // [2][wavefront][gate, up][value][lane]
    int count, share, lines, tiles;
    int step_at, step_tile;
    struct Place {
        int at, tile;
    } opening, closing_at;

    __device__ GateUp(const FewArgs &l, const FewLists &lists, float *red, int cls, int who, int shares) : l(l), lists(lists), red(red)
    {
        tiles = (l.F + 15) / 16;
        lines = (l.H + Form::kLineCols - 1) / Form::kLineCols;
        share = (lines + kFewWaves - 1) / kFewWaves;
        const int begin = __builtin_amdgcn_readfirstlane(lists.begin[cls]), end = __builtin_amdgcn_readfirstlane(lists.begin[cls + 1]);
        // items are numbered through all classes; those of a share are `shares` apart
        const int skip = (int)((unsigned)begin * (unsigned)tiles % (unsigned)shares), first = who >= skip ? who - skip : who - skip + shares;
        const int items = (end - begin) * tiles;
        count = first < items ? (items - 1 - first) / shares + 1 : 0;
        opening = closing_at = {begin + first / tiles, first % tiles};
        step_at = shares / tiles;
        step_tile = shares % tiles;
    }
    __device__ __forceinline__ void advance(Place &p) const
    {
        p.at += step_at;
        p.tile += step_tile;
        if (p.tile >= tiles)
            p.tile -= tiles, ++p.at;
    }
    __device__ __forceinline__ int segments() const { return count; }
    __device__ __forceinline__ int length(int) const { return share; }
    __device__ __forceinline__ bool ready() const { return true; }
    __device__ __forceinline__ void open(FewCursor<kForm, kTT, 2> &c, int)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int expert = __builtin_amdgcn_readfirstlane(lists.expert[opening.at]), base = __builtin_amdgcn_readfirstlane(lists.base[opening.at]);
        const int rows = __builtin_amdgcn_readfirstlane(lists.rows[opening.at]);
        const int64_t row = (int64_t)expert * l.F + opening.tile * 16, end = (int64_t)(expert + 1) * l.F;
        c.panel[0] = panel_of<kForm>(l.gate, row, end, l.H, l.scale_cols_h);
        c.panel[1] = panel_of<kForm>(l.up, row, end, l.H, l.scale_cols_h);
        const uint32_t x_row = (uint32_t)l.H * Form::kElt;
        c.set_acts({static_cast<const unsigned char *>(l.x), (uint32_t)l.N * x_row, 16 * Form::kElt, rows},
                   [&](int r) { return lists.token[base + r] * x_row; });
        c.line = wave * share;
        c.left = share;
        c.lines = lines;
        advance(opening);
    }
    __device__ __forceinline__ void close(const FewSums<kForm, kTT, 2> &sums, int k)
    {
        constexpr int kValues = kFewValues<kForm, kTT>;
        const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        float *const mine = red + (k % 2) * (kFewWaves * 2 * kValues * kWave);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int v = 0; v < kValues; ++v)
                mine[((wave * 2 + c) * kValues + v) * kWave + lane] = sums.value(c, v);
        few_barrier(); // (the other half's readers were done before its writers came here)
        const int at = closing_at.at, f0 = closing_at.tile * 16;
        advance(closing_at);
        for (int v = (wave + k) % kFewWaves; v < kValues; v += kFewWaves) {
            float total[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                total[c] = mine[(c * kValues + v) * kWave + lane];
#pragma unroll
                for (int w = 1; w < kFewWaves; ++w)
                    total[c] += mine[((w * 2 + c) * kValues + v) * kWave + lane];
            }
            const float a = silu_mul_f32(total[0], total[1]);
            const int base = __builtin_amdgcn_readfirstlane(lists.base[at]), rows = __builtin_amdgcn_readfirstlane(lists.rows[at]);
            const FewActs to = few_activation<kForm>(l, base, rows);
            const int r = few_row_of<kForm, kTT>(v), i = lane % 16;
            const bool there = r < rows && f0 + i < l.F;
            unsigned char *const tile = const_cast<unsigned char *>(to.data) + (int64_t)(f0 / 16) * to.tile + (r * 16 + i) * Form::kElt;
            if constexpr (kForm == kFewF32) {
                if (there)
                    __hip_atomic_store(reinterpret_cast<uint32_t *>(tile), __float_as_uint(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            } else { // the even lane stores both columns (F is even)
                const uint32_t both = pack_bf16x2(a, __shfl_xor(a, 1));
                if (there && lane % 2 == 0)
                    __hip_atomic_store(reinterpret_cast<uint32_t *>(tile), both, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
    }
};

// A class's part of a down tile, columns [h0, h0 + cols): the experts' lines side by side are shared by the wavefronts, whose
// weighted rows are added to their own sums per token.
template <int kForm, int kTT, int kCT, class Ready>
struct Down {
    using Form = FewForm<kForm>;
    const FewArgs &l;
    const FewLists &lists;
    float *token_sums;
    int h0, cols;
    Ready wait;
    int lines, begin, from, to;

    __device__ Down(const FewArgs &l, const FewLists &lists, float *token_sums, int cls, int h0, int cols, Ready wait)
        : l(l), lists(lists), token_sums(token_sums), h0(h0), cols(cols), wait(wait)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        lines = (l.F + Form::kLineCols - 1) / Form::kLineCols;
        begin = __builtin_amdgcn_readfirstlane(lists.begin[cls]);
        const int64_t all = (int64_t)(__builtin_amdgcn_readfirstlane(lists.begin[cls + 1]) - begin) * lines;
        from = (int)(all * wave / kFewWaves);
        to = (int)(all * (wave + 1) / kFewWaves);
    }
    __device__ __forceinline__ int segments() const { return to > from ? (to - 1) / lines - from / lines + 1 : 0; }
    __device__ __forceinline__ int first_line(int k) const { return k ? 0 : from % lines; }
    __device__ __forceinline__ int length(int k) const
    {
        const int start = k ? (from / lines + k) * lines : from, end = (from / lines + k + 1) * lines;
        return (end < to ? end : to) - start;
    }
    __device__ __forceinline__ bool ready() { return wait(); }
    __device__ __forceinline__ void open(FewCursor<kForm, kTT, kCT> &c, int k)
    {
        const int at = begin + from / lines + k;
        const int expert = __builtin_amdgcn_readfirstlane(lists.expert[at]), base = __builtin_amdgcn_readfirstlane(lists.base[at]);
        const int rows = __builtin_amdgcn_readfirstlane(lists.rows[at]);
        const int64_t row = (int64_t)expert * l.H + h0, end = row + cols;
#pragma unroll
        for (int p = 0; p < kCT; ++p)
            c.panel[p] = panel_of<kForm>(l.down, row + 16 * p, end, l.F, l.scale_cols_f);
        c.set_acts(few_activation<kForm>(l, base, rows), [&](int r) { return (uint32_t)(r * 16 * Form::kElt); });
        c.line = first_line(k);
        c.left = length(k);
        c.lines = lines;
    }
    __device__ __forceinline__ void close(const FewSums<kForm, kTT, kCT> &sums, int k)
    {
        const int at = begin + from / lines + k;
        const int base = __builtin_amdgcn_readfirstlane(lists.base[at]), rows = __builtin_amdgcn_readfirstlane(lists.rows[at]);
#pragma unroll
        for (int v = 0; v < kFewValues<kForm, kTT>; ++v) {
            const int r = few_row_of<kForm, kTT>(v);
            if (r < rows) { // (a token has an expert once: the lanes of a wavefront meet nowhere)
                const float w = lists.weight[base + r];
                float *const to_sum = token_sums + lists.token[base + r] * (16 * kCT) + threadIdx.x % 16;
#pragma unroll
                for (int p = 0; p < kCT; ++p)
                    to_sum[16 * p] += w * sums.value(p, v);
            }
        }
    }
};
#endif

// kMaxTT: sixteens of rows that an expert can have (N).  kCT: sixteens of columns of a down tile.
template <int kForm, int kMaxTT, int kCT>
__global__ __launch_bounds__(kFewThreads, 2) void few_ffn(FewKernelArgs g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kRed = 2 * kFewWaves * 2 * (kMaxTT > 1 ? 4 * kMaxTT : 4) * kWave, kSums = kFewWaves * 16 * kMaxTT * 16 * kCT;
    __shared__ union {
        FewRouting routing;
        float red[kRed];
        float sums[kSums];
    } sh;
    __shared__ FewLists lists;
    __shared__ int box[kFewWaves];
    const FewArgs &l = g.l;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    for (int e = threadIdx.x; e < l.E; e += kFewThreads)
        sh.routing.mask[e] = 0;
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
        const int groups = (l.N + kFewWaves - 1) / kFewWaves;
        for (int who = (int)blockIdx.x < groups ? (int)blockIdx.x : -1;;) {
            if (who >= 0) {
                const int n = who * kFewWaves + wave;
                if (n < l.N) {
                    const Pick p = few_select(g, n);
                    if (lane < l.K) {
                        __hip_atomic_store(l.topk_idx + n * l.K + lane, p.expert, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        __hip_atomic_store(l.topk_w + n * l.K + lane, p.weight, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    }
                }
                few_signal(g.flags + who);
            }
            who = few_missing(g.flags, groups, g.patience, box);
            if (who < 0)
                break;
        }
        for (int p = threadIdx.x; p < l.N * l.K; p += kFewThreads) {
            sh.routing.pick[p] = (uint16_t)__hip_atomic_load(l.topk_idx + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            sh.routing.weight[p] = __hip_atomic_load(l.topk_w + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    __syncthreads();
    few_make_lists<kForm>(lists, sh.routing, l.N, l.K, l.E);

    uint32_t *const share_flags = g.flags + 32;
    const FewCols in = {l.H, l.scale_cols_h, l.group}, mid = {l.F, l.scale_cols_f, l.group};
    bool all_there = false;
    for (int who = blockIdx.x;;) {
        auto gate_up = [&](auto tt, int cls) {
            constexpr int kTT = decltype(tt)::value;
            GateUp<kForm, kTT> items(l, lists, sh.red, cls, who, g.shares);
            few_stream<kForm, kTT, 2, few_depth<kForm, kTT, 2>()>(items, in);
            few_barrier(); // (the next one writes red)
        };
        gate_up(std::integral_constant<int, 0>{}, 0);
        gate_up(std::integral_constant<int, 1>{}, 1);
        if constexpr (kMaxTT > 1) {
            gate_up(std::integral_constant<int, 2>{}, 2);
            gate_up(std::integral_constant<int, 4>{}, 3);
        }
        few_signal(share_flags + who);

        int missing = -1;
        const int tile = l.N * 16 * kCT;
        float *const mine = sh.sums + wave * tile;
        for (int h0 = (int)blockIdx.x * g.down_cols; h0 < l.H && missing < 0; h0 += (int)gridDim.x * g.down_cols) {
            for (int p = lane; p < tile; p += kWave)
                mine[p] = 0.0f;
            const int cols = l.H - h0 < g.down_cols ? l.H - h0 : g.down_cols;
            auto wait = [&]() {
                if (!all_there) {
                    missing = few_missing(share_flags, g.shares, g.patience, box);
                    all_there = missing < 0;
                }
                return all_there;
            };
            auto down = [&](auto tt, int cls) {
                constexpr int kTT = decltype(tt)::value;
                if (missing >= 0 || __builtin_amdgcn_readfirstlane(lists.begin[cls]) == __builtin_amdgcn_readfirstlane(lists.begin[cls + 1]))
                    return;
                Down<kForm, kTT, kCT, decltype(wait)> part(l, lists, mine, cls, h0, cols, wait);
                few_stream<kForm, kTT, kCT, few_depth<kForm, kTT, kCT>()>(part, mid);
            };
            down(std::integral_constant<int, 0>{}, 0);
            down(std::integral_constant<int, 1>{}, 1);
            if constexpr (kMaxTT > 1) {
                down(std::integral_constant<int, 2>{}, 2);
                down(std::integral_constant<int, 4>{}, 3);
            }
            if (missing >= 0)
                break;
            few_barrier();
            for (int p = threadIdx.x * 2; p < tile; p += kFewThreads * 2) { // (columns are even)
                float v[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    v[u] = sh.sums[p + u];
#pragma unroll
                    for (int w = 1; w < kFewWaves; ++w)
                        v[u] += sh.sums[w * tile + p + u];
                }
                const int n = p / (16 * kCT), h = p % (16 * kCT);
                if (h < cols) {
                    if constexpr (kForm == kFewF32)
                        *reinterpret_cast<f32x2 *>(static_cast<float *>(l.out) + (int64_t)n * l.H + h0 + h) = f32x2{v[0], v[1]};
                    else
                        *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(l.out) + (int64_t)n * l.H + h0 + h) = pack_bf16x2(v[0], v[1]);
                }
            }
            few_barrier(); // (the sums are written again)
        }
        if (missing < 0)
            return;
        few_barrier();
        who = missing;
    }
#endif
}

template <int kForm>
void launch_few_ffn(const FewKernelArgs &g, hipStream_t st)
{
    const dim3 grid((unsigned)g.shares), block(kFewThreads);
    if (g.l.N <= 16) {
        if (g.down_cols <= 16)
            hipLaunchKernelGGL((few_ffn<kForm, 1, 1>), grid, block, 0, st, g);
        else
            hipLaunchKernelGGL((few_ffn<kForm, 1, 2>), grid, block, 0, st, g);
    } else {
        if (g.down_cols <= 16)
            hipLaunchKernelGGL((few_ffn<kForm, 4, 1>), grid, block, 0, st, g);
        else
            hipLaunchKernelGGL((few_ffn<kForm, 4, 2>), grid, block, 0, st, g);
    }
}

extern template void launch_few_ffn<kFewBf16>(const FewKernelArgs &g, hipStream_t st);
extern template void launch_few_ffn<kFewF32>(const FewKernelArgs &g, hipStream_t st);
extern template void launch_few_ffn<kFewFp4>(const FewKernelArgs &g, hipStream_t st);
extern template void launch_few_ffn<kFewInt4>(const FewKernelArgs &g, hipStream_t st);

}  // namespace moe

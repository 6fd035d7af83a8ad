// The whole layer for a few tokens, in two launches.
//
//   few_logits   router logits, each as eight partial sums; clears the flags of the second launch; for 4-bit weights, x in the
//                operands' order
//   few_ffn      top-K, expert lists, both products of the experts that got a row, the weighted sum
//
// The layer is bound by reading the touched experts' weights once (16 tokens of 256 experts of 7168 x 2048, bf16: 6.0 TB/s), with
// 4 bits also by what few_stream.h says; everything else is latency (one token of 4 experts, 35 us in all: logits 5, top-K and
// lists 3, gate/up 8 - 12, the flags 2, down 6, sums 3).  few_ffn has one workgroup
// per compute unit, with a fixed share of each step:
//   tokens   (more than few_route_all says) top-K of eight tokens, one per wavefront; of fewer every workgroup selects for
//            itself, which is quicker than waiting for another's answer
//   gate/up  items (expert, a few columns of F): both products of the expert's rows and the activation, into the workspace
//   down     a few columns of H over ALL touched experts (as many as make a share for every workgroup): a token's sum over
//            its K experts is made in one workgroup, in ascending k, so there is no third exchange
// Within a workgroup the wavefronts draw their work, items or parts of items, from counters in LDS: served unequally by the
// memory, they would wait for each other a fifth of the time otherwise.  What is added up, and in which order, does not depend
// on who draws what: partial sums meet in LDS and are added by their place, so equal calls give equal bits.
// Shares of workgroups are fixed because drawing them costs more than it gives: atomics on one address in memory are served
// one in 12 ns (512 workgroups that drew from one counter and polled another: one token 64 us instead of 27).
//
// What a step needs from other workgroups is said by a flag per share.  A workgroup that has waited for longer than any share
// takes does a missing share itself (a second time, with the same bits, if its owner is only late), and another one as long as
// one is missing, without a wait between them: every wait ends, however few workgroups of the grid are resident, several calls
// on several streams included.  Workgroups that wait take different shares (the first missing one, the second, ..., by their own
// number), so that together they need about missing / waiting turns (3 tokens, H = 192: 0.11 ms with 100 of 256 workgroups).
// The activation goes from XCD to XCD.  It is written through and a share's flag is set once its stores are acknowledged.  It
// is read by ordinary loads: a cache line belongs to one item, so no XCD can hold one that was read or written in part before
// its item was complete.  (Telling the caches to drop what they hold takes 5 - 9 us.)
//
// Rows of an expert are the set bits of a mask of 64 tokens: slot and count are population counts, in ascending n.  Experts are
// taken in three classes by their rows (few_stream.h's forms), each a stream of its own.
#pragma once

#include <math.h>

#include "common.h"
#include "few.h"
#include "few_stream.h"
#include "select.h"

namespace moe {

constexpr int kParts = 8; // partial sums of a logit between the launches
constexpr int kMaxTokens = MOE_FEW_TOKENS, kMaxRows = kMaxTokens * (int)MOE_MAX_TOPK;
constexpr int kMaxShares = 1024, kFlags = 32 + kMaxShares; // tokens', then shares'

// ------------------------------------------------------------------------
struct FewKernelArgs {
    FewArgs l;
    const float *parts;
    const void *x; // as gate/up reads it: packed for 4-bit weights
    int x_cols;    // of a row of it
    uint32_t *flags;
    int workgroups;
    int shares;    // of gate/up items
    int width;      // columns of F of an item: 8 or 16
    int down_cols;  // columns of H of a down tile, at most 16 kCT
    int down_parts; // of an expert's reduction there
    int patience; // polls of a wait
    int h_lines, f_lines, f_tiles; // lines of H and F; items of an expert
};

constexpr int kPoolFloats = 32768; // LDS for partial sums

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

// One token per wavefront, or two where a lane has one logit (9 tokens of 16 experts 28.6 -> 27.5 us, 16 of 64 48.1 -> 47.4; but
// 16 of 256 51.7 -> 53.1, three per wavefront 24 of 32 38.7 -> 38.8).
__device__ __forceinline__ bool few_route_all(const FewArgs &l) { return l.N <= (l.E <= kWave ? 2 : 1) * kFewWaves; }

// The experts that got a row, by class and in ascending order within it, and their rows: slots from base on.  An expert with
// more than a stream's rows (N K / 33 experts at most) is there twice: with that many, and with the rest.
constexpr int kMaxEntries = MOE_MAX_EXPERTS + kMaxRows / 33;
struct FewLists {
    int begin[4]; // of the classes: at most kFewRows rows, 16, 32
    uint16_t expert[kMaxEntries], base[kMaxEntries];
    uint16_t lines[kMaxEntries]; // cache lines of one activation tile before this one's
    uint8_t rows[kMaxEntries];
    uint8_t token[kMaxRows]; // of a slot
    uint16_t slot[kMaxRows]; // of n * K + k, and its weight
    float weight[kMaxRows];
};
struct FewRouting { // while the lists are made
    uint64_t mask[MOE_MAX_EXPERTS];  // of tokens
    uint16_t first[MOE_MAX_EXPERTS]; // slot
    uint16_t pick[kMaxRows];
    float weight[kMaxRows];
    uint64_t wave_sum[kFewWaves];
    uint32_t wave_rows[kFewWaves];
};

// An expert's activation: tiles of `width` columns; a tile is its rows side by side, in whole cache lines.
template <int kForm>
__device__ __forceinline__ uint32_t few_tile_lines(int rows, int width)
{
    return (uint32_t)(rows * width * FewForm<kForm>::kElt + 127) / 128u;
}

// All threads; r.pick and r.weight are there, r.mask is zero.
template <int kForm>
__device__ __forceinline__ void few_make_lists(FewLists &lists, FewRouting &r, int N, int K, int E, int width)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    for (int at = threadIdx.x; at < N * K; at += kFewThreads)
        atomicOr(reinterpret_cast<unsigned long long *>(&r.mask[r.pick[at]]), 1ull << (at / K));
    __syncthreads();
    // Two experts per thread.  Sums: cache lines of a tile in the low 13 bits, then experts of each class in 11 bits; slots.
    constexpr int kPer = MOE_MAX_EXPERTS / kFewThreads;
    auto shift_of = [](int rows) { return 13 + 11 * (rows <= FewForm<kForm>::kFewRows ? 0 : rows <= 16 ? 1 : 2); };
    uint64_t mine[kPer], up_to = 0;
    uint32_t slots = 0;
    int rows[kPer];
    auto entry = [&](int rows) { return rows ? (uint64_t)few_tile_lines<kForm>(rows, width) | 1ull << shift_of(rows) : 0; };
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = threadIdx.x * kPer + i;
        rows[i] = e < E ? (int)__popcll(r.mask[e]) : 0;
        mine[i] = rows[i] <= kFewMost ? entry(rows[i]) : entry(kFewMost) + entry(rows[i] - kFewMost);
        up_to += mine[i];
        slots += rows[i];
    }
    uint64_t at = 0 - up_to, all = 0;
    uint32_t slot = 0u - slots;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        const uint64_t v = __shfl_up((unsigned long long)up_to, s);
        const uint32_t u = __shfl_up(slots, s);
        up_to += lane >= s ? v : 0;
        slots += lane >= s ? u : 0u;
    }
    if (lane == kWave - 1) {
        r.wave_sum[wave] = up_to;
        r.wave_rows[wave] = slots;
    }
    __syncthreads();
    at += up_to;
    slot += slots;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        at += w < wave ? r.wave_sum[w] : 0;
        slot += w < wave ? r.wave_rows[w] : 0u;
        all += r.wave_sum[w];
    }
    int begin[4] = {0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < 3; ++c)
        begin[c + 1] = begin[c] + (int)(all >> (13 + 11 * c) & 0x7FF);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = threadIdx.x * kPer + i;
        uint64_t here = at;
        for (int done = 0; done < rows[i];) {
            const int some = rows[i] - done < kFewMost ? rows[i] - done : kFewMost, shift = shift_of(some);
            const int place = (shift == 13 ? 0 : shift == 24 ? begin[1] : begin[2]) + (int)(here >> shift & 0x7FF);
            lists.expert[place] = (uint16_t)e;
            lists.rows[place] = (uint8_t)some;
            lists.lines[place] = (uint16_t)(here & 0x1FFF);
            lists.base[place] = (uint16_t)(slot + done);
            here += entry(some);
            done += some;
        }
        if (rows[i])
            r.first[e] = (uint16_t)slot;
        at += mine[i];
        slot += rows[i];
    }
    if (threadIdx.x == 0)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            lists.begin[c] = begin[c];
    __syncthreads();
    for (int p = threadIdx.x; p < N * K; p += kFewThreads) {
        const int e = r.pick[p], n = p / K;
        const int s = r.first[e] + (int)__popcll(r.mask[e] & ((1ull << n) - 1));
        lists.token[s] = (uint8_t)n;
        lists.slot[p] = (uint16_t)s;
        lists.weight[p] = r.weight[p];
    }
    __syncthreads();
}

// All threads: -1 once all flags are set; if some still are not after `patience` polls, one of them: of m, the one that has
// blockIdx.x % m before it.  After that `patience` is 0.  box: of at least count / 64 + 1.
__device__ __forceinline__ int few_missing(const uint32_t *flags, int count, int &patience, uint64_t *box)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, words = (count + kWave - 1) / kWave;
    for (int poll = 0;; ++poll) {
        for (int c = wave; c < words; c += kFewWaves) {
            const int i = c * kWave + lane;
            const uint64_t miss = __ballot(i < count && __hip_atomic_load(flags + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0);
            if (lane == 0)
                box[c] = miss;
        }
        few_barrier();
        const bool some = __ballot(lane < words && box[lane] != 0) != 0;
        int found = -1;
        if (some && poll >= patience) {
            int m = 0;
            for (int c = 0; c < words; ++c)
                m += (int)__popcll(box[c]);
            int before = (int)(blockIdx.x % (uint32_t)m);
            for (int c = 0; c < words && found < 0; ++c) {
                uint64_t left = box[c];
                const int here = (int)__popcll(left);
                if (before < here) {
                    for (; before > 0; --before)
                        left &= left - 1;
                    found = c * kWave + (int)__builtin_ctzll(left);
                }
                before -= here;
            }
            patience = 0;
        }
        found = __builtin_amdgcn_readfirstlane(found);
        few_barrier();
        if (!some || found >= 0)
            return found;
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

// The activation of the expert at place `at`.
template <int kForm>
__device__ __forceinline__ FewActs few_activation(const FewKernelArgs &g, const FewLists &lists, int at, int rows)
{
    const uint32_t lines = __builtin_amdgcn_readfirstlane(lists.lines[at]), tiles = (uint32_t)g.f_tiles;
    const uint32_t tile = few_tile_lines<kForm>(rows, g.width) * 128u;
    return {static_cast<const unsigned char *>(g.l.a) + (int64_t)lines * tiles * 128, tiles * tile, g.width, tile, rows};
}

// Gate/up items of one class: (expert, `width` columns of F); a share's are `shares` apart.  A unit, which a wavefront draws,
// is an item or a part of its reduction.
template <int kForm, int kTT>
struct GateUp {
    using Form = FewForm<kForm>;
    static constexpr int kCT = 2, kDepth = few_depth<kForm, kTT, kCT>(); // tiles: gate, up
    static constexpr int kValues = kFewValues<kForm, kTT>, kActs = Form::kQ4 ? kActPacked : kActRows;
    const FewKernelArgs &g;
    const FewArgs &l;
    const FewLists &lists;
    float *pool;
    FewRoom &room;
    int *counter;
    int begin, items, first, mine, parts;
    struct Unit {
        int n, at, tile, part; // n-th item of the share
    } open_unit, unit;
    bool any = false;

    // before: items of the classes before this one (items are numbered through all classes); it is moved on
    __device__ GateUp(const FewKernelArgs &g, const FewLists &lists, float *pool, FewRoom &room, int *counter, int cls, int who, int &before)
        : g(g), l(g.l), lists(lists), pool(pool), room(room), counter(counter)
    {
        begin = __builtin_amdgcn_readfirstlane(lists.begin[cls]);
        items = (__builtin_amdgcn_readfirstlane(lists.begin[cls + 1]) - begin) * g.f_tiles;
        first = who - (before ? before % g.shares : 0);
        if (first < 0)
            first += g.shares;
        mine = first < items ? (items - 1 - first) / g.shares + 1 : 0;
        before += items;
        parts = __builtin_amdgcn_readfirstlane(few_parts(mine, g.h_lines, kDepth));
    }
    __device__ __forceinline__ bool open(FewCursor<kForm, kTT, kCT, kActs> &c)
    {
        const int u = few_draw(counter);
        if (u >= mine * parts)
            return false;
        const int n = u / parts, item = first + n * g.shares, at = begin + item / g.f_tiles, f0 = item % g.f_tiles * g.width;
        open_unit = {n, at, item % g.f_tiles, u % parts};
        if (!any)
            unit = open_unit;
        any = true;
        const int expert = __builtin_amdgcn_readfirstlane(lists.expert[at]), base = __builtin_amdgcn_readfirstlane(lists.base[at]);
        const int rows = __builtin_amdgcn_readfirstlane(lists.rows[at]);
        const int64_t row = (int64_t)expert * l.F + f0, end = row + (l.F - f0 < g.width ? l.F - f0 : g.width);
        c.panel[0] = panel_of<kForm>(l.gate, row, end, l.H, l.scale_cols_h);
        c.panel[1] = panel_of<kForm>(l.up, row, end, l.H, l.scale_cols_h);
        const uint32_t x_row = (uint32_t)g.x_cols * Form::kElt;
        c.set_acts({static_cast<const unsigned char *>(g.x), (uint32_t)l.N * x_row, 0, 0, rows},
                   [&](int r) { return lists.token[base + r] * x_row; });
        c.line = few_part_line<kForm>(g.h_lines, open_unit.part, parts);
        c.end = few_part_line<kForm>(g.h_lines, open_unit.part + 1, parts);
        c.groups = c.end > c.line ? (c.end - c.line + kDepth - 1) / kDepth : 1;
        return true;
    }
    // Value v of the lanes.  In bf16 the activation is rounded to bf16 here, as moe_grouped_ffn rounds it: it is the down product's
    // operand (a second number for the rest would double its loads and products), and a prompt's tokens and the next ones go
    // through the same roundings.
    __device__ __forceinline__ void store(int v, float gate, float up) const
    {
        const float a = silu_mul_f32(gate, up);
        const int rows = __builtin_amdgcn_readfirstlane(lists.rows[unit.at]);
        const FewActs to = few_activation<kForm>(g, lists, unit.at, rows);
        const int r = few_row_of<kForm, kTT>(v), i = threadIdx.x % 16;
        const bool there = r < rows && i < g.width && unit.tile * g.width + i < l.F;
        const int col = i % 8;
        unsigned char *const put = const_cast<unsigned char *>(to.data) + (int64_t)unit.tile * to.tile + (i / 8 * rows + r) * (8 * Form::kElt);
        if constexpr (kForm == kFewF32) {
            if (there)
                __hip_atomic_store(reinterpret_cast<uint32_t *>(put) + col, __float_as_uint(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        } else { // one lane stores two columns (F and width are even): neighbours, or (INT4) those that int4_order has side by side
            constexpr int kOther = Form::kInt4 ? 2 : 1;
            const int place = Form::kInt4 ? col / 4 + col % 2 * 2 : col / 2;
            const uint32_t both = pack_bf16x2(a, __shfl_xor(a, kOther));
            if (there && (threadIdx.x & kOther) == 0)
                __hip_atomic_store(reinterpret_cast<uint32_t *>(put) + place, both, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    __device__ __forceinline__ void close(const FewSums<kForm, kTT, kCT> &sums)
    {
        if (parts == 1) {
#pragma unroll
            for (int v = 0; v < kValues; ++v)
                store(v, sums.value(0, v), sums.value(1, v));
        } else {
            FewJoin<kForm, kTT, kCT>(pool, kPoolFloats, room, parts).close(sums, unit.n, unit.part, [&](auto total) {
                for (int v = 0; v < kValues; ++v)
                    store(v, total(0, v), total(1, v));
            });
        }
        unit = open_unit;
    }
};

// All threads: the first weights of a down tile, columns [h0, h0 + cols) of the experts in their order, are asked for: kAhead cache
// lines per thread, to be in L2 when the activation is complete (one token 35.6 -> 34.8 us, fp4 36.9 -> 36.0).  What is read is
// nobody's result.
constexpr int kAhead = 2;
template <int kForm>
__device__ __forceinline__ void few_ask_ahead(const FewKernelArgs &g, const FewLists &lists, int h0, int cols, uint32_t got[kAhead])
{
    constexpr int kScaleBytes = kForm == kFewFp4 ? 1 : 2;
    const FewArgs &l = g.l;
    const uint32_t bytes = (uint32_t)(cols * FewForm<kForm>::row_bytes(l.F)), scale_bytes = FewForm<kForm>::kQ4 ? cols * l.scale_cols_f * kScaleBytes : 0;
    const uint32_t lines = (bytes + 127) / 128, each = lines + (scale_bytes + 127) / 128;
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
        const uint32_t u = a * kFewThreads + threadIdx.x, at = u / each, line = u % each;
        got[a] = 0;
        if (at < (uint32_t)lists.begin[3]) {
            const int64_t row = (int64_t)lists.expert[at] * l.H + h0;
            if (line < lines)
                got[a] = (static_cast<const unsigned char *>(l.down.data) + row * FewForm<kForm>::row_bytes(l.F))[line * 128];
            else
                got[a] = (static_cast<const unsigned char *>(l.down.scales) + row * l.scale_cols_f * kScaleBytes)[(line - lines) * 128];
        }
    }
}

// A class's part of a down tile, columns [h0, h0 + cols).  A unit is one of `down_parts` parts of an expert's reduction; its
// rows go to LDS by part and slot.
template <int kForm, int kTT, int kCT>
struct Down {
    using Form = FewForm<kForm>;
    static constexpr int kDepth = few_depth<kForm, kTT, kCT>();
    const FewKernelArgs &g;
    const FewArgs &l;
    const FewLists &lists;
    float *pool; // [part][slot][16 kCT]
    int *counter;
    int h0, cols;
    int begin, units;
    struct Unit {
        int at, part;
    } open_unit, unit;
    bool any = false;

    __device__ Down(const FewKernelArgs &g, const FewLists &lists, float *pool, int *counter, int cls, int h0, int cols)
        : g(g), l(g.l), lists(lists), pool(pool), counter(counter), h0(h0), cols(cols)
    {
        begin = __builtin_amdgcn_readfirstlane(lists.begin[cls]);
        units = (__builtin_amdgcn_readfirstlane(lists.begin[cls + 1]) - begin) * g.down_parts;
    }
    __device__ __forceinline__ bool open(FewCursor<kForm, kTT, kCT, kActTiles> &c)
    {
        const int u = few_draw(counter);
        if (u >= units)
            return false;
        const int at = begin + u / g.down_parts;
        open_unit = {at, u % g.down_parts};
        if (!any)
            unit = open_unit;
        any = true;
        const int expert = __builtin_amdgcn_readfirstlane(lists.expert[at]), rows = __builtin_amdgcn_readfirstlane(lists.rows[at]);
        const int64_t row = (int64_t)expert * l.H + h0, end = row + cols;
#pragma unroll
        for (int p = 0; p < kCT; ++p)
            c.panel[p] = panel_of<kForm>(l.down, row + 16 * p, end, l.F, l.scale_cols_f);
        c.set_acts(few_activation<kForm>(g, lists, at, rows), [](int r) { return r * (8u * Form::kElt); });
        c.line = few_part_line<kForm>(g.f_lines, open_unit.part, g.down_parts);
        c.end = few_part_line<kForm>(g.f_lines, open_unit.part + 1, g.down_parts);
        c.groups = c.end > c.line ? (c.end - c.line + kDepth - 1) / kDepth : 1;
        return true;
    }
    __device__ __forceinline__ void close(const FewSums<kForm, kTT, kCT> &sums)
    {
        const int base = __builtin_amdgcn_readfirstlane(lists.base[unit.at]), rows = __builtin_amdgcn_readfirstlane(lists.rows[unit.at]);
        float *const to = pool + (unit.part * l.N * l.K + base) * (16 * kCT) + threadIdx.x % 16;
#pragma unroll
        for (int v = 0; v < kFewValues<kForm, kTT>; ++v) {
            const int r = few_row_of<kForm, kTT>(v);
            if (r < rows)
#pragma unroll
                for (int p = 0; p < kCT; ++p)
                    to[r * (16 * kCT) + 16 * p] = sums.value(p, v);
        }
        unit = open_unit;
    }
};
#endif

// kMaxTT: sixteens of rows that an entry of the lists can have.  kCT: sixteens of columns of a down tile.
template <int kForm, int kMaxTT, int kCT>
__global__ __launch_bounds__(kFewThreads, 2) void few_ffn(FewKernelArgs g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ union {
        FewRouting routing;
        float pool[kPoolFloats];
    } sh;
    __shared__ FewLists lists;
    __shared__ FewRoom room;
    __shared__ int counters[3]; // units drawn, of each class
    __shared__ uint64_t box[kMaxShares / kWave];
    const FewArgs &l = g.l;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    for (int e = threadIdx.x; e < l.E; e += kFewThreads)
        sh.routing.mask[e] = 0;
    if (few_route_all(l)) {
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
        int patience = g.patience;
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
            who = few_missing(g.flags, groups, patience, box);
            if (who < 0)
                break;
        }
        for (int p = threadIdx.x; p < l.N * l.K; p += kFewThreads) {
            sh.routing.pick[p] = (uint16_t)__hip_atomic_load(l.topk_idx + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            sh.routing.weight[p] = __hip_atomic_load(l.topk_w + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    __syncthreads();
    few_make_lists<kForm>(lists, sh.routing, l.N, l.K, l.E, g.width);

    uint32_t *const share_flags = g.flags + 32;
    const FewCols in = {l.H, l.scale_cols_h}, mid = {l.F, l.scale_cols_f};
    auto restart = [&]() { // of the counters; everyone is done with them
        if (threadIdx.x < 3)
            counters[threadIdx.x] = 0;
        if (threadIdx.x < 8) {
            room.parts_done[threadIdx.x] = 0;
            room.item[threadIdx.x] = threadIdx.x;
        }
        few_barrier();
    };
    auto empty = [&](int cls) { return __builtin_amdgcn_readfirstlane(lists.begin[cls]) == __builtin_amdgcn_readfirstlane(lists.begin[cls + 1]); };
    int patience = g.patience;
    for (int who = blockIdx.x;;) {
        int before = 0;
        restart();
        auto gate_up = [&](auto tt, int cls) {
            constexpr int kTT = decltype(tt)::value;
            if (empty(cls))
                return;
            using Items = GateUp<kForm, kTT>;
            Items items(g, lists, sh.pool, room, counters + cls, cls, who, before);
            few_stream<kForm, kTT, Items::kCT, Items::kDepth, Items::kActs>(items, in);
            if (items.parts > 1) { // (the next class has other places in the pool)
                few_barrier();
                restart();
            }
        };
        gate_up(std::integral_constant<int, 0>{}, 0);
        gate_up(std::integral_constant<int, 1>{}, 1);
        if constexpr (kMaxTT > 1)
            gate_up(std::integral_constant<int, 2>{}, 2);
        few_signal(share_flags + who);
        const int h0 = (int)blockIdx.x * g.down_cols;
        if (h0 >= l.H)
            return;
        uint32_t got[kAhead];
        few_ask_ahead<kForm>(g, lists, h0, l.H - h0 < g.down_cols ? l.H - h0 : g.down_cols, got);
        who = few_missing(share_flags, g.shares, patience, box);
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            asm volatile("" ::"v"(got[a])); // (the loads are wanted)
        if (who < 0)
            break;
    }

    for (int h0 = (int)blockIdx.x * g.down_cols; h0 < l.H; h0 += (int)gridDim.x * g.down_cols) {
        const int cols = l.H - h0 < g.down_cols ? l.H - h0 : g.down_cols;
        restart();
        auto down = [&](auto tt, int cls) {
            constexpr int kTT = decltype(tt)::value;
            if (empty(cls))
                return;
            using Part = Down<kForm, kTT, kCT>;
            Part part(g, lists, sh.pool, counters + cls, cls, h0, cols);
            few_stream<kForm, kTT, kCT, Part::kDepth, kActTiles>(part, mid);
        };
        down(std::integral_constant<int, 0>{}, 0);
        down(std::integral_constant<int, 1>{}, 1);
        if constexpr (kMaxTT > 1)
            down(std::integral_constant<int, 2>{}, 2);
        few_barrier();
        for (int p = threadIdx.x * 2; p < l.N * 16 * kCT; p += kFewThreads * 2) { // (columns are even)
            const int n = p / (16 * kCT), h = p % (16 * kCT);
            if (h >= cols)
                continue;
            float v[2] = {0.0f, 0.0f};
            for (int k = 0; k < l.K; ++k) {
                const float w = lists.weight[n * l.K + k];
                const float *from = sh.pool + lists.slot[n * l.K + k] * (16 * kCT) + h;
                float y[2] = {from[0], from[1]};
                for (int part = 1; part < g.down_parts; ++part) {
                    from += l.N * l.K * (16 * kCT);
                    y[0] += from[0];
                    y[1] += from[1];
                }
                v[0] += w * y[0];
                v[1] += w * y[1];
            }
            if constexpr (kForm == kFewF32)
                *reinterpret_cast<f32x2 *>(static_cast<float *>(l.out) + (int64_t)n * l.H + h0 + h) = f32x2{v[0], v[1]};
            else
                *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(l.out) + (int64_t)n * l.H + h0 + h) = pack_bf16x2(v[0], v[1]);
        }
        few_barrier(); // (the pool is written again)
    }
#endif
}

template <int kForm>
void launch_few_ffn(const FewKernelArgs &g, hipStream_t st)
{
    const dim3 grid((unsigned)g.workgroups), block(kFewThreads);
    if (g.l.N <= 16) {
        if (g.down_cols <= 16)
            hipLaunchKernelGGL((few_ffn<kForm, 1, 1>), grid, block, 0, st, g);
        else
            hipLaunchKernelGGL((few_ffn<kForm, 1, 2>), grid, block, 0, st, g);
    } else {
        if (g.down_cols <= 16)
            hipLaunchKernelGGL((few_ffn<kForm, 2, 1>), grid, block, 0, st, g);
        else
            hipLaunchKernelGGL((few_ffn<kForm, 2, 2>), grid, block, 0, st, g);
    }
}

extern template void launch_few_ffn<kFewBf16>(const FewKernelArgs &g, hipStream_t st);
extern template void launch_few_ffn<kFewF32>(const FewKernelArgs &g, hipStream_t st);
extern template void launch_few_ffn<kFewFp4>(const FewKernelArgs &g, hipStream_t st);
extern template void launch_few_ffn<kFewInt4By32>(const FewKernelArgs &g, hipStream_t st);
extern template void launch_few_ffn<kFewInt4By64>(const FewKernelArgs &g, hipStream_t st);
extern template void launch_few_ffn<kFewInt4By128>(const FewKernelArgs &g, hipStream_t st);

}  // namespace moe

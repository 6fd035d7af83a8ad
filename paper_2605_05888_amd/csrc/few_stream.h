// Products of a few rows with a panel of weight rows, as a stream of weights: what the decoding operators are made of.
//
// With a handful of rows a product is bound by reading the weights.  A wavefront reads lines of 64 (4 bits) or 128 bytes of
// sixteen weight rows at a time, straight into registers in the operand layout of the matrix instructions, with kDepth
// lines in flight; the activations of the same columns come beside them, from L2.  The matrix instructions are the cheap
// part (an eighth of the time a line takes to arrive), also where most of their rows are empty.
//
// The weights are the instruction's second operand, the activations the first: lane (q, i) = (lane / 16, lane % 16) holds
// eight (fp32: four) columns of weight row i, and register r of a result belongs to activation row 4 q + r and weight row i.
// Which columns of a line a lane holds is free as long as both operands agree.  A line has kChunks chunks, one operand
// each; chunk t of lane q are the columns
//   bf16   32 t +  8 q ..   two 16-byte loads per line, four lanes side by side read 64 bytes
//   fp32   16 t +  4 q ..   (four instructions of four columns each per chunk)
//   FP4    32 q +  8 t ..   one 16-byte load: a lane has a whole group of 32 columns, so it needs one scale byte, which the
//                           conversion to bf16 multiplies in (a power of two: exact)
//   INT4   32 t +  8 q ..   one 16-byte load of columns 32 q .., then a transposition between the four lanes: an instruction
//                           then covers one group of 32 columns, and the scale is applied to its sum in fp32.  A code c is
//                           the bf16 number 128 + c (a byte beside 0x43); 136 times the sum of the activations, which an
//                           instruction with ones gives, is subtracted.  (A weight times its scale would have to be rounded.)
//
// kTT > 0: up to 16 kTT rows.  Row 16 tt + i of the activations is in lane i, kChunks loads per line and 16 rows.
// kTT = 0: at most 16 / kChunks rows (kFewRows), one load per line: lane i holds chunk i % kChunks of row i / kChunks.  The
// instruction of chunk t then gives sense only in result rows i with i % kChunks == t, and every chunk has a result of its own:
// with four chunks, register t of result t in lane q is row q's.  (An expert of a decoded batch mostly has that few rows.
// Four times fewer loads and registers for the activations of 4-bit weights, and for INT4 one multiplication per scale.)
#pragma once

#include "common.h"
#include "few.h"
#include "q4.h"

namespace moe {

// How a weight matrix is held; activations are bf16 but for kFewF32.
enum { kFewBf16 = 0, kFewF32 = 1, kFewFp4 = 2, kFewInt4 = 3 };

template <int kForm>
struct FewForm {
    static constexpr bool kQ4 = kForm == kFewFp4 || kForm == kFewInt4;
    static constexpr int kElt = kForm == kFewF32 ? 4 : 2;                        // bytes of an activation
    static constexpr int kLineCols = kQ4 ? 128 : kForm == kFewF32 ? 32 : 64;     // columns of a line
    static constexpr int kLineBytes = kQ4 ? 64 : 128;                            // of a weight row
    static constexpr int kLoads = kQ4 ? 1 : 2;                                   // 16-byte loads of a line per lane
    static constexpr int kChunks = kQ4 ? 4 : 2;
    static constexpr int kFewRows = 16 / kChunks;
    static constexpr bool kRagged = kForm != kFewBf16;                           // the last line may be cut short
    __host__ __device__ static constexpr int64_t row_bytes(int64_t cols) { return kQ4 ? cols / 2 : cols * kElt; }
};

constexpr uint32_t kNowhere = 0x80000000u; // an offset past every byte count used here: loads give zeros

#if defined(__HIP_DEVICE_COMPILE__)

// Sixteen weight rows.  bytes: of those that are there; scales: from the first row's first scale, scale_bytes as bytes.
struct Panel {
    const unsigned char *data, *scales;
    uint32_t bytes, scale_bytes;
};

// Rows [row, row + 16) of matrix w, whose rows end at `rows`; nothing if row is past that.
template <int kForm>
__device__ __forceinline__ Panel panel_of(const FewMatrix &w, int64_t row, int64_t rows, int cols, int scale_cols)
{
    const int there = (int)(rows - row < 16 ? (rows > row ? rows - row : 0) : 16);
    const int64_t at = there ? row : 0, row_bytes = FewForm<kForm>::row_bytes(cols);
    Panel p;
    p.data = static_cast<const unsigned char *>(w.data) + at * row_bytes;
    p.bytes = (uint32_t)(there * row_bytes);
    p.scales = nullptr;
    p.scale_bytes = 0;
    if constexpr (FewForm<kForm>::kQ4) {
        constexpr int kBytes = kForm == kFewFp4 ? 1 : 2;
        p.scales = static_cast<const unsigned char *>(w.scales) + at * scale_cols * kBytes;
        p.scale_bytes = (uint32_t)(there * scale_cols * kBytes);
    }
    return p;
}

// Where the activations of a segment are: row r, column c at row_of(r) + c / 16 * tile + c % 16 elements, all below `bytes`.
// (Row-major matrices: tile is sixteen elements.)
struct FewActs {
    const unsigned char *data;
    uint32_t bytes;
    uint32_t tile; // bytes
    int rows;
};

struct FewCols {
    int cols, scale_cols;
    int group; // of INT4
};

// Values a lane ends up with per weight row, and the activation row of value v.
template <int kForm, int kTT>
constexpr int kFewValues = kTT ? 4 * kTT : 4 / FewForm<kForm>::kChunks;
template <int kForm, int kTT>
__device__ __forceinline__ int few_row_of(int v)
{
    const int q = threadIdx.x % kWave / 16;
    return kTT ? 16 * (v / 4) + 4 * q + v % 4 : kFewValues<kForm, 0> * q + v;
}

template <int kForm, int kTT, int kCT>
struct FewOperands {
    static constexpr int kRows = kTT ? kTT : 1, kActs = kTT ? FewForm<kForm>::kChunks : 1;
    u32x4 w[kCT][FewForm<kForm>::kLoads];
    uint32_t scale[kCT];
    u32x4 a[kRows][kActs];
};

template <int kForm, int kTT, int kCT>
struct FewSums {
    static constexpr int kRows = kTT ? kTT : 1;
    static constexpr bool kScalar = kForm == kFewInt4 && kTT == 0;
    static constexpr int kParts = kTT ? 1 : FewForm<kForm>::kChunks;
    f32x4 acc[kScalar ? 1 : kRows][kScalar ? 1 : kCT][kScalar ? 1 : kParts];
    float one[kScalar ? kCT : 1];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int c = 0; c < kCT; ++c) {
            if constexpr (kScalar)
                one[c] = 0.0f;
            else
#pragma unroll
                for (int t = 0; t < kRows; ++t)
#pragma unroll
                    for (int p = 0; p < kParts; ++p)
                        acc[t][c][p] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
    // value v of weight row tile c
    __device__ __forceinline__ float value(int c, int v) const
    {
        if constexpr (kScalar)
            return one[c];
        else if constexpr (kTT > 0)
            return acc[v / 4][c][0][v % 4];
        else if constexpr (kParts == 4)
            return (acc[0][c][0][0] + acc[0][c][1][1]) + (acc[0][c][2][2] + acc[0][c][3][3]);
        else
            return acc[0][c][0][2 * v] + acc[0][c][1][2 * v + 1];
    }
};

// Eight FP4 codes as bf16 times their scale.
__device__ __forceinline__ bf16x8 fp4_operand(uint32_t codes, float scale)
{
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return __builtin_bit_cast(bf16x8, r);
}

// Eight INT4 codes as bf16 numbers 128 + c, in the order of columns 0, 2, 4, 6, 1, 3, 5, 7 (int4_order gives the
// activations the same).
__device__ __forceinline__ bf16x8 int4_operand(uint32_t codes)
{
    const uint32_t even = codes & 0x0F0F0F0Fu, odd = (codes >> 4) & 0x0F0F0F0Fu, high = 0x43434343u;
    // byte selectors 0 - 3: of the second operand, 4 - 7: of the first
    const u32x4 r = {__builtin_amdgcn_perm(high, even, 0x04010400u), __builtin_amdgcn_perm(high, even, 0x04030402u),
                     __builtin_amdgcn_perm(high, odd, 0x04010400u), __builtin_amdgcn_perm(high, odd, 0x04030402u)};
    return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ bf16x8 int4_order(u32x4 a)
{
    const u32x4 r = {__builtin_amdgcn_perm(a[1], a[0], 0x05040100u), __builtin_amdgcn_perm(a[3], a[2], 0x05040100u),
                     __builtin_amdgcn_perm(a[1], a[0], 0x07060302u), __builtin_amdgcn_perm(a[3], a[2], 0x07060302u)};
    return __builtin_bit_cast(bf16x8, r);
}

// Registers w[j] of four lanes q with the same i, transposed: w[j] of lane q becomes what w[q] was in lane j.
__device__ __forceinline__ u32x4 transpose_quads(u32x4 w)
{
    const auto a = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false);
    const auto b = __builtin_amdgcn_permlane16_swap(w[2], w[3], false, false);
    const auto c = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false);
    const auto d = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
    return u32x4{c[0], d[0], c[1], d[1]};
}

template <int kForm, int kTT, int kCT>
__device__ __forceinline__ void few_multiply(FewSums<kForm, kTT, kCT> &sums, const FewOperands<kForm, kTT, kCT> &o, int group)
{
    using Form = FewForm<kForm>;
    using Ops = FewOperands<kForm, kTT, kCT>;
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (kForm == kFewF32) {
#pragma unroll
        for (int t = 0; t < Form::kChunks; ++t)
#pragma unroll
            for (int c = 0; c < kCT; ++c)
#pragma unroll
                for (int m = 0; m < Ops::kRows; ++m) {
                    f32x4 &acc = sums.acc[m][c][kTT ? 0 : t];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(o.a[m][kTT ? t : 0][j]),
                                                                   __uint_as_float(o.w[c][t][j]), acc, 0, 0, 0);
                }
    } else if constexpr (kForm != kFewInt4) {
#pragma unroll
        for (int c = 0; c < kCT; ++c) {
            const float scale = kForm == kFewFp4 ? fp4_scale(o.scale[c]) : 0.0f;
#pragma unroll
            for (int t = 0; t < Form::kChunks; ++t) {
                bf16x8 w;
                if constexpr (kForm == kFewFp4)
                    w = fp4_operand(o.w[c][0][t], scale);
                else
                    w = __builtin_bit_cast(bf16x8, o.w[c][t]);
#pragma unroll
                for (int m = 0; m < Ops::kRows; ++m) {
                    f32x4 &acc = sums.acc[m][c][kTT ? 0 : t];
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, o.a[m][kTT ? t : 0]), w, acc, 0, 0, 0);
                }
            }
        }
    } else {
        const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
        // the scales of the line's four groups of 32 columns, for every lane q
        float scale[kCT][4];
        u32x4 w[kCT];
#pragma unroll
        for (int c = 0; c < kCT; ++c) {
            const uint32_t s = o.scale[c] << 16;
            const auto pair = __builtin_amdgcn_permlane16_swap(s, s, false, false);
            const auto even = __builtin_amdgcn_permlane32_swap(pair[0], pair[0], false, false);
            const auto odd = __builtin_amdgcn_permlane32_swap(pair[1], pair[1], false, false);
            scale[c][0] = __uint_as_float(even[0]), scale[c][2] = __uint_as_float(even[1]);
            scale[c][1] = __uint_as_float(odd[0]), scale[c][3] = __uint_as_float(odd[1]);
            w[c] = transpose_quads(o.w[c][0]);
        }
        if constexpr (kTT == 0) {
            const bf16x8 a = int4_order(o.a[0][0]);
            const f32x4 sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, ones, zero, 0, 0, 0);
#pragma unroll
            for (int c = 0; c < kCT; ++c)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const f32x4 d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, int4_operand(w[c][t]), zero, 0, 0, 0);
                    sums.one[c] = fmaf(scale[c][t], fmaf(-136.0f, sum[t], d[t]), sums.one[c]);
                }
        } else {
            auto chained = [&](auto groups) { // of 32 columns under one scale
                constexpr int kSame = decltype(groups)::value;
#pragma unroll
                for (int t = 0; t < 4; t += kSame)
#pragma unroll
                    for (int m = 0; m < Ops::kRows; ++m) {
                        bf16x8 a[kSame];
                        f32x4 sum = zero;
#pragma unroll
                        for (int u = 0; u < kSame; ++u) {
                            a[u] = int4_order(o.a[m][kTT ? t + u : 0]);
                            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[u], ones, sum, 0, 0, 0);
                        }
#pragma unroll
                        for (int c = 0; c < kCT; ++c) {
                            f32x4 d = zero;
#pragma unroll
                            for (int u = 0; u < kSame; ++u)
                                d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[u], int4_operand(w[c][t + u]), d, 0, 0, 0);
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                sums.acc[m][c][0][r] = fmaf(scale[c][t], fmaf(-136.0f, sum[r], d[r]), sums.acc[m][c][0][r]);
                        }
                    }
            };
            if (group == 32)
                chained(std::integral_constant<int, 1>{});
            else if (group == 64)
                chained(std::integral_constant<int, 2>{});
            else
                chained(std::integral_constant<int, 4>{});
        }
    }
}

// The part of the stream that the next line is fetched from: panels and activations of one segment, for this lane.
template <int kForm, int kTT, int kCT>
struct FewCursor {
    using Form = FewForm<kForm>;
    static constexpr int kRows = kTT ? kTT : 1, kActs = kTT ? Form::kChunks : 1;
    Panel panel[kCT];
    const unsigned char *act;
    uint32_t act_bytes, act_line; // act_line: bytes from one line's activations to the next one's
    uint32_t row_off[kRows], chunk_off[kActs];
    int line, left, lines; // next line, lines left of this wavefront's, lines of a row

    // first column of chunk t of this lane's line
    static __device__ __forceinline__ int chunk_col(int t)
    {
        const int q = threadIdx.x % kWave / 16;
        return kForm == kFewFp4 ? 32 * q + 8 * t : (Form::kLineCols / Form::kChunks) * t + (16 / Form::kElt) * q;
    }
    template <class RowOf>
    __device__ __forceinline__ void set_acts(const FewActs &a, RowOf row_of)
    {
        const int i = threadIdx.x % 16;
        act = a.data;
        act_bytes = a.bytes;
        act_line = (uint32_t)(Form::kLineCols / 16) * a.tile;
#pragma unroll
        for (int m = 0; m < kRows; ++m) {
            const int r = kTT ? 16 * m + i : i / Form::kChunks;
            row_off[m] = r < a.rows ? row_of(r) : kNowhere;
        }
#pragma unroll
        for (int t = 0; t < kActs; ++t) {
            const int col = chunk_col(kTT ? t : i % Form::kChunks);
            chunk_off[t] = (uint32_t)(col / 16) * a.tile + (uint32_t)(col % 16 * Form::kElt);
        }
    }
};

// A wavefront's stream: segment after segment (a panel of weight rows with the activation rows that meet it, some lines of
// both), without a gap in the loads between them.  The source says what they are:
//   segments()            how many
//   length(k)             lines of segment k, at least 1 (lines past the row's end read as zeros)
//   open(cursor, k)       sets the cursor to segment k; k ascending, kDepth lines ahead of
//   close(sums, k)        takes the sums of segment k
//   ready()               called once, when the first weights are under way and before the first activations are asked for;
//                         false: there are none, the stream ends
template <int kForm, int kTT, int kCT, int kDepth, class Source>
__device__ __forceinline__ void few_stream(Source &source, const FewCols &g)
{
    using Form = FewForm<kForm>;
    using Ops = FewOperands<kForm, kTT, kCT>;
    using Cursor = FewCursor<kForm, kTT, kCT>;
    const int segments = source.segments();
    if (segments == 0) {
        (void)source.ready();
        return;
    }
    const int lane = threadIdx.x % kWave, i = lane % 16, q = lane / 16;
    const uint32_t w_off = (uint32_t)i * (uint32_t)Form::row_bytes(g.cols) + (uint32_t)q * 16u;
    const int scale_off = i * g.scale_cols;
    const int group_shift = kForm == kFewInt4 ? (g.group == 32 ? 0 : g.group == 64 ? 1 : 2) : 0;
    auto fetch_weights = [&](Ops &o, const Cursor &c) {
        const bool there = c.line < c.lines; // (else no bytes: zeros, and the number of loads in flight stays)
#pragma unroll
        for (int p = 0; p < kCT; ++p) {
            const auto rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(c.panel[p].data), 0,
                                                              there ? (int)c.panel[p].bytes : 0, 0x00020000);
#pragma unroll
            for (int s = 0; s < Form::kLoads; ++s) // (weights are read once: non-temporal)
                o.w[p][s] = __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(w_off + (uint32_t)(c.line * Form::kLineBytes + 64 * s)), 0, 2);
            if constexpr (Form::kQ4) {
                const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(c.panel[p].scales), 0,
                                                                  there ? (int)c.panel[p].scale_bytes : 0, 0x00020000);
                const int at = scale_off + ((c.line * 4 + q) >> group_shift);
                if constexpr (kForm == kFewFp4)
                    o.scale[p] = __builtin_amdgcn_raw_buffer_load_b8(rs, at, 0, 0);
                else
                    o.scale[p] = __builtin_amdgcn_raw_buffer_load_b16(rs, 2 * at, 0, 0);
            }
        }
    };
    auto fetch_acts = [&](Ops &o, const Cursor &c) {
        const bool there = c.line < c.lines;
        const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(c.act), 0, there ? (int)c.act_bytes : 0, 0x00020000);
        const uint32_t base = (uint32_t)c.line * c.act_line;
        const int col0 = c.line * Form::kLineCols;
#pragma unroll
        for (int t = 0; t < Ops::kActs; ++t) {
            // columns past the row's end would be another row's
            const bool in = !Form::kRagged || col0 + Cursor::chunk_col(kTT ? t : i % Form::kChunks) < g.cols;
#pragma unroll
            for (int m = 0; m < Ops::kRows; ++m)
                o.a[m][t] = __builtin_amdgcn_raw_buffer_load_b128(ra, (int)(in ? c.row_off[m] + c.chunk_off[t] + base : kNowhere), 0, 0);
        }
    };
    Cursor c;
    int opened = 0; // segments
    auto open = [&]() {
        if (opened < segments) {
            source.open(c, opened);
            ++opened;
        } else {
            c.lines = 0; // nothing more
            c.left = 0x7FFFFFFF;
        }
    };
    auto advance = [&]() {
        ++c.line;
        if (--c.left == 0)
            open();
        // one order of the loads everywhere: else the wait at the top of the loop is for all of them
        __builtin_amdgcn_sched_barrier(0);
    };
    Ops o[kDepth];
    {
        // The weights of the first lines go out before ready(), their activations after it.
        Cursor starts[kDepth];
        open();
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            starts[d] = c;
            fetch_weights(o[d], c);
            advance();
        }
        if (!source.ready())
            return;
#pragma unroll
        for (int d = 0; d < kDepth; ++d)
            fetch_acts(o[d], starts[d]);
        __builtin_amdgcn_sched_barrier(0);
    }
    FewSums<kForm, kTT, kCT> sums;
    sums.clear();
    int closing = 0, left = source.length(0);
    for (;;) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            few_multiply(sums, o[d], g.group);
            __builtin_amdgcn_sched_barrier(0);
            if (--left == 0) {
                source.close(sums, closing);
                if (++closing == segments)
                    return;
                sums.clear();
                left = source.length(closing);
            }
            fetch_weights(o[d], c);
            fetch_acts(o[d], c);
            advance();
        }
    }
}

// LDS and register barrier without the memory fence of __syncthreads, which would wait for the loads in flight.
__device__ __forceinline__ void few_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
#endif

}  // namespace moe

// Products of a few rows with a panel of weight rows, as a stream of weights: what the decoding operators are made of.
//
// With a handful of rows a product is bound by reading the weights.  A wavefront reads lines of 64 (4 bits) or 128 bytes of
// sixteen weight rows at a time, straight into registers, with kDepth lines in flight; the activations of the same columns come
// beside them, from L2.  In bf16 that runs at what panels of sixteen rows can be read with (5.4 - 6.2 TB/s, one large read 6.7).
// With 4 bits there are four times as many products, conversions and activations per byte, and they take about as long as the
// reading: 37 tokens of 32 experts fp4 take 165 us, 135 without the activations and scales, 106 without the weights.
//
// The weights are the matrix instruction's second operand, the activations the first: lane (q, i) = (lane / 16, lane % 16) holds
// eight (fp32: four) columns of weight row i, and register r of a result belongs to activation row 4 q + r and weight row i.
// Which columns of a line a lane holds is free as long as both operands agree.  A line has kChunks chunks, one operand
// each; chunk t of lane q are the columns
//   bf16   32 t +  8 q ..   two 16-byte loads per line
//   fp32   16 t +  4 q ..   (four instructions of four columns each per chunk)
//   4 bits one 16-byte load holds columns 32 q ..; with activations in the same order (kOwn: 32 q + 8 t ..) that is it.  A group
//          of 32 or 64 columns under one INT4 scale has to be in one instruction (32 t + 8 q ..), and so have activations in
//          the caller's order: then four lanes transpose what they have.
// FP4 codes become bf16 numbers times their scale on the way (a power of two: exact).  INT4: the scale is applied to an
// instruction's sum in fp32 (a weight times its scale would have to be rounded).  A code c becomes the bf16 number c 2^-12, so an
// instruction starts from -8 2^-12 times the sum of the activations, which another one gives: sums hold up to 15 and 8 scales
// of a weight that is at most 8.  (c - 8 itself takes seven instructions more for eight codes: 8 tokens of 256 experts 268 ->
// 318 us.)  With the 2^-12, which the whole sum takes back at its end, 128 columns of the largest activations have finite sums.
// Scales are loaded for four lines at once, lane q those of line q: a load costs the address unit the same sixteen rows
// whether it fetches a byte a row or sixteen (a byte per lane and line: the unit was busy 0.73 of the time).
//
// kTT > 0: up to 16 kTT rows.  Row 16 tt + i of the activations is in lane i, kChunks loads per line and 16 rows.
// kTT = 0: at most 16 / kChunks rows (kFewRows), one load per line: lane i holds chunk i % kChunks of row i / kChunks.  The
// instruction of chunk t then gives sense only in result rows i with i % kChunks == t, and every chunk has a result of its own:
// with four chunks, register t of result t in lane q is row q's.  (An expert of a decoded batch mostly has that few rows.
// Four times fewer loads and registers for the activations of 4-bit weights, and for INT4 one multiplication per scale.)
//
// In that layout neighbouring lanes hold different rows, and the address unit takes a load of sixteen bytes a lane four
// neighbouring lanes at a time: 64 bytes of one line in a cycle, or four lines in four (fetched like that, the unit was busy
// 0.6 - 0.8 of the time).  So lane l fetches what lane (l % 4, l / 4) of the layout needs, four neighbours 64 bytes of a row,
// and the registers change lanes on arrival (ds_bpermute).
//
// No register may be spilled: the compiler loses lanes of one that is (build.py refuses it), which sets the depths.
#pragma once

#include "common.h"
#include "few.h"
#include "q4.h"

namespace moe {

// How a weight matrix is held; activations are bf16 but for kFewF32.
// (INT4: by the columns of a scale.)
enum { kFewBf16 = 0, kFewF32 = 1, kFewFp4 = 2, kFewInt4By32 = 3, kFewInt4By64 = 4, kFewInt4By128 = 5 };

template <int kForm>
struct FewForm {
    static constexpr bool kInt4 = kForm >= kFewInt4By32, kQ4 = kForm == kFewFp4 || kInt4;
    static constexpr int kSame = kForm == kFewInt4By128 ? 4 : kForm == kFewInt4By64 ? 2 : 1; // groups of 32 columns under one scale
    static constexpr int kElt = kForm == kFewF32 ? 4 : 2;                        // bytes of an activation
    static constexpr int kLineCols = kQ4 ? 128 : kForm == kFewF32 ? 32 : 64;     // columns of a line
    static constexpr int kLineBytes = kQ4 ? 64 : 128;                            // of a weight row
    static constexpr int kLoads = kQ4 ? 1 : 2;                                   // 16-byte loads of a line per lane
    static constexpr int kChunks = kQ4 ? 4 : 2;
    static constexpr int kFewRows = 16 / kChunks;
    static constexpr bool kRagged = kForm != kFewBf16;                           // the last line may be cut short
    static constexpr bool kOwn = kForm == kFewFp4 || kForm == kFewInt4By128;     // packed: a lane's columns of a line are its own
    __host__ __device__ static constexpr int64_t row_bytes(int64_t cols) { return kQ4 ? cols / 2 : cols * kElt; }
};

constexpr int kFewWaves = 8, kFewThreads = kFewWaves * kWave; // of a workgroup
constexpr int kFewMost = 32; // rows of a stream: what 256 registers hold
// How the activations of a stream are laid out: rows as the caller has them; rows, or tiles, as the operands want them.
enum { kActRows, kActPacked, kActTiles };

constexpr uint32_t kNowhere = 0x40000000u; // an offset past every byte count used here, twice too: loads give zeros

#if defined(__HIP_DEVICE_COMPILE__)

// A buffer of `bytes` bytes at p.  Both are the same in all lanes; the compiler, which cannot see it everywhere, would else
// load lane by lane in a loop.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t few_buffer(const void *p, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    const uint64_t low = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at);
    const uint64_t high = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(high << 32 | low), 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}

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

// Where the activations of a segment are, all below `bytes`: rows at row_of(r), or tiles of `width` columns (8 or 16), `tile`
// bytes apart: in a tile eight columns of all rows, then the other eight.
struct FewActs {
    const unsigned char *data;
    uint32_t bytes;
    int width;
    uint32_t tile;
    int rows;
};

struct FewCols {
    int cols, scale_cols;
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
    u32x4 a[kRows][kActs];
};

constexpr float kInt4Unit = 0x1p-12f; // of INT4 operands

template <int kForm, int kTT, int kCT>
struct FewSums {
    static constexpr int kRows = kTT ? kTT : 1;
    static constexpr bool kScalar = FewForm<kForm>::kInt4 && kTT == 0;
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
            return one[c] * (1.0f / kInt4Unit);
        else if constexpr (FewForm<kForm>::kInt4)
            return acc[v / 4][c][0][v % 4] * (1.0f / kInt4Unit);
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

// Eight INT4 codes as bf16 numbers c kInt4Unit, in the order of columns 0, 2, 4, 6, 1, 3, 5, 7 (int4_order gives the
// activations the same).  A byte from 0 to 15 is that many 2^-9 as an e4m3 number.
__device__ __forceinline__ bf16x8 int4_operand(uint32_t codes)
{
    const uint32_t even = codes & 0x0F0F0F0Fu, odd = codes >> 4 & 0x0F0F0F0Fu;
    constexpr float scale = kInt4Unit * 0x1p9f;
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, scale, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, scale, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, scale, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, scale, true));
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

// Scales of four lines: as loaded (lane q: those of line q, FP4 four bytes, INT4 up to four bf16), and for every lane.
template <int kForm, int kCT>
struct FewScales {
    static constexpr int kRegs = kForm == kFewInt4By32 ? 2 : 1;
    uint32_t raw[kCT][kRegs];
    uint32_t shift[kCT]; // bits that a load was moved back by, so as not to pass the panel's end
    uint32_t keep[kRegs]; // of the segment: past it may be another row's, an infinity or NaN, which times zero is not zero
    uint32_t of[kCT][4][kRegs];

    // own: of an FP4 line a lane needs the scale of its own group only
    template <bool kOwn>
    __device__ __forceinline__ void spread()
    {
        const int row = (int)(threadIdx.x % 16) * 16; // byte address of the lane that fetched line 0's of row i
        const int mine = (int)(threadIdx.x % kWave / 16) * 8;
#pragma unroll
        for (int c = 0; c < kCT; ++c) {
            if constexpr (kRegs == 2) {
                const uint64_t v = ((uint64_t)raw[c][1] << 32 | raw[c][0]) >> (shift[c] & 63);
                raw[c][0] = (uint32_t)v & keep[0], raw[c][1] = (uint32_t)(v >> 32) & keep[1];
            } else {
                raw[c][0] = raw[c][0] >> shift[c] & keep[0];
            }
#pragma unroll
            for (int r = 0; r < kRegs; ++r)
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    uint32_t v = (uint32_t)__builtin_amdgcn_ds_bpermute(row + 4 * d, (int)raw[c][r]);
                    if constexpr (kOwn && kForm == kFewFp4)
                        v = v >> mine & 0xFFu;
                    of[c][d][r] = v;
                }
        }
    }
    // of the columns of instruction t in line d (0 .. 3)
    template <bool kOwn>
    __device__ __forceinline__ float fp4(int c, int d, int t) const
    {
        return fp4_scale(kOwn ? of[c][d][0] : of[c][d][0] >> (8 * t) & 0xFFu);
    }
    __device__ __forceinline__ float int4(int c, int d, int place) const
    {
        const uint32_t v = of[c][d][kRegs == 2 ? place / 2 : 0];
        return __uint_as_float(place % 2 ? v & 0xFFFF0000u : v << 16);
    }
};

// Two lines of a panel that were fetched as its upper and its lower eight rows, each 128 bytes (32 lanes the first 64 of all,
// 32 the others): as lines.
template <int kForm, int kTT, int kCT>
__device__ __forceinline__ void few_to_lines(FewOperands<kForm, kTT, kCT> &first, FewOperands<kForm, kTT, kCT> &second)
{
#pragma unroll
    for (int c = 0; c < kCT; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const auto v = __builtin_amdgcn_permlane32_swap(first.w[c][0][j], second.w[c][0][j], false, false);
            first.w[c][0][j] = v[0], second.w[c][0][j] = v[1];
        }
}

// What a lane has fetched, to the lane whose operand it is.
__device__ __forceinline__ void from_lane(u32x4 &v, int from)
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        v[j] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * from, (int)v[j]);
}

template <int kForm, int kTT, int kCT, int kActs>
__device__ __forceinline__ void to_operand_lanes(FewOperands<kForm, kTT, kCT> &o)
{
    using Form = FewForm<kForm>;
    const int i = (int)(threadIdx.x % 16), q = (int)(threadIdx.x % kWave / 16);
#pragma unroll
    for (int c = 0; c < kCT; ++c)
#pragma unroll
        for (int l = 0; l < Form::kLoads; ++l)
            from_lane(o.w[c][l], 4 * i + q);
    if constexpr (kActs != kActTiles) {
#pragma unroll
        for (int m = 0; m < FewOperands<kForm, kTT, kCT>::kRows; ++m)
#pragma unroll
            for (int t = 0; t < FewOperands<kForm, kTT, kCT>::kActs; ++t)
                from_lane(o.a[m][t], 4 * i + q);
    } else if constexpr (kTT == 0) {
        const int t = i % Form::kChunks, piece = Form::kOwn ? Form::kChunks * q + t : 4 * t + q;
        from_lane(o.a[0][0], piece * Form::kFewRows + i / Form::kChunks);
    }
}

// Line d of four.
template <int kForm, int kTT, int kCT, int kActs>
__device__ __forceinline__ void few_multiply(FewSums<kForm, kTT, kCT> &sums, const FewOperands<kForm, kTT, kCT> &o,
                                             const FewScales<kForm, kCT> &scales, int d)
{
    using Form = FewForm<kForm>;
    using Ops = FewOperands<kForm, kTT, kCT>;
    constexpr bool kPacked = kActs != kActRows, kOwn = kPacked && Form::kOwn;
    auto words = [&](int c) { return kOwn ? o.w[c][0] : transpose_quads(o.w[c][0]); }; // of the instructions
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
    } else if constexpr (!Form::kInt4) {
        u32x4 codes[kCT];
        if constexpr (kForm == kFewFp4)
#pragma unroll
            for (int c = 0; c < kCT; ++c)
                codes[c] = words(c);
#pragma unroll
        for (int t = 0; t < Form::kChunks; ++t)
#pragma unroll
            for (int c = 0; c < kCT; ++c) {
                bf16x8 w;
                if constexpr (kForm == kFewFp4)
                    w = fp4_operand(codes[c][t], scales.template fp4<kOwn>(c, d, t));
                else
                    w = __builtin_bit_cast(bf16x8, o.w[c][t]);
#pragma unroll
                for (int m = 0; m < Ops::kRows; ++m) {
                    f32x4 &acc = sums.acc[m][c][kTT ? 0 : t];
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, o.a[m][kTT ? t : 0]), w, acc, 0, 0, 0);
                }
            }
    } else {
        // -8 units times the activations' sum is where an instruction starts from
        constexpr int kSame = Form::kSame;
        static_assert(kInt4Unit == 0x1p-12f);
        const bf16x8 minus = __builtin_bit_cast(bf16x8, u32x4{0xBB00BB00u, 0xBB00BB00u, 0xBB00BB00u, 0xBB00BB00u}); // -2^-9
        auto act = [&](const u32x4 &a) { return kPacked ? __builtin_bit_cast(bf16x8, a) : int4_order(a); };
        if constexpr (kTT == 0) {
            const bf16x8 a = act(o.a[0][0]);
            const f32x4 sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, minus, zero, 0, 0, 0);
#pragma unroll
            for (int c = 0; c < kCT; ++c) {
                const u32x4 codes = words(c);
                float v[4];
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    v[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, int4_operand(codes[t]), sum, 0, 0, 0)[t];
#pragma unroll
                for (int t = 0; t < 4; t += kSame) {
                    float all = v[t];
#pragma unroll
                    for (int u = 1; u < kSame; ++u)
                        all += v[t + u];
                    sums.one[c] = fmaf(scales.int4(c, d, t / kSame), all, sums.one[c]);
                }
            }
        } else {
            u32x4 codes[kCT];
#pragma unroll
            for (int c = 0; c < kCT; ++c)
                codes[c] = words(c);
#pragma unroll
            for (int t = 0; t < 4; t += kSame) {
                bf16x8 w[kCT][kSame];
#pragma unroll
                for (int c = 0; c < kCT; ++c)
#pragma unroll
                    for (int u = 0; u < kSame; ++u)
                        w[c][u] = int4_operand(codes[c][t + u]);
#pragma unroll
                for (int m = 0; m < Ops::kRows; ++m) {
                    f32x4 sum = zero, p[kCT];
#pragma unroll
                    for (int u = 0; u < kSame; ++u)
                        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(act(o.a[m][t + u]), minus, sum, 0, 0, 0);
#pragma unroll
                    for (int c = 0; c < kCT; ++c)
                        p[c] = sum;
#pragma unroll
                    for (int u = 0; u < kSame; ++u)
#pragma unroll
                        for (int c = 0; c < kCT; ++c)
                            p[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(act(o.a[m][t + u]), w[c][u], p[c], 0, 0, 0);
#pragma unroll
                    for (int c = 0; c < kCT; ++c) {
                        const float scale = scales.int4(c, d, t / kSame);
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            sums.acc[m][c][0][r] = fmaf(scale, p[c][r], sums.acc[m][c][0][r]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    }
}

// Where the stream's next lines are fetched from: panels and activations of one segment, for this lane.
template <int kForm, int kTT, int kCT, int kActs>
struct FewCursor {
    using Form = FewForm<kForm>;
    static constexpr int kRows = kTT ? kTT : 1;
    static constexpr int kPiece = 16 / Form::kElt; // columns of a load
    Panel panel[kCT];
    const unsigned char *act;
    uint32_t act_bytes, act_tile, act_eight, act_wide; // eight: bytes of eight columns; wide: a tile has 16 columns (1) or 8 (0)
    uint32_t row_off[kRows];
    int line, end, groups; // next line, the segment's last, groups of kDepth lines left

    // Row r of sixteens m of the activations that this lane fetches, and the first column in the line of its load t.  Rows:
    // four neighbours 64 bytes of one.  Tiles: as many neighbours as there are rows the same columns.
    static __device__ __forceinline__ int lane_row(int m)
    {
        const int lane = threadIdx.x % kWave;
        if constexpr (kActs == kActTiles)
            return kTT ? 16 * m + lane % 16 : lane % Form::kFewRows;
        return kTT ? 16 * m + lane / 4 : lane / 4 / Form::kChunks;
    }
    static __device__ __forceinline__ int lane_col(int t)
    {
        const int lane = threadIdx.x % kWave;
        if constexpr (kActs == kActTiles)
            return kPiece * (kTT == 0 ? lane / Form::kFewRows : Form::kOwn ? Form::kChunks * (lane / 16) + t : 4 * t + lane / 16);
        return Form::kLineCols / Form::kChunks * (kTT ? t : lane / 4 % Form::kChunks) + kPiece * (lane % 4);
    }
    template <class RowOf>
    __device__ __forceinline__ void set_acts(const FewActs &a, RowOf row_of)
    {
        act = a.data;
        act_bytes = a.bytes;
        if constexpr (kActs == kActTiles) {
            act_tile = a.tile;
            act_eight = (uint32_t)a.rows * (8u * Form::kElt);
            act_wide = a.width == 16;
        }
#pragma unroll
        for (int m = 0; m < kRows; ++m) {
            const int r = lane_row(m);
            row_off[m] = r < a.rows ? row_of(r) : kNowhere;
        }
    }
    // Byte offset of a column in its row.
    __device__ __forceinline__ uint32_t col_off(int col) const
    {
        if constexpr (kActs != kActTiles)
            return (uint32_t)(col * Form::kElt);
        const uint32_t n = (uint32_t)col / 8u;
        return (n >> act_wide) * act_tile + (n & act_wide) * act_eight + (uint32_t)(col % 8 * Form::kElt);
    }
};

// Lines in flight per wavefront: what 256 registers hold beside a line's products (registers of a line in the comment).
template <int kForm, int kTT, int kCT>
constexpr int few_depth()
{
    if (FewForm<kForm>::kQ4) // 4 kCT + 4, 16, 32
        return kTT == 0 ? (FewForm<kForm>::kInt4 && kCT == 2 ? 4 : 8) : kTT == 1 ? 4 : 2;
    return kTT <= 1 ? (kCT == 1 ? 8 : 4) : kCT == 1 ? 4 : 3; // 8 kCT + 4, 8, 16
}

// 4-bit lines are half a cache line.  Where there is depth for it they are fetched in pairs, eight rows of 128 bytes a load: a
// cache line that is asked for by two loads, the second before it has arrived, holds both up (8 tokens of 256 experts int4
// 289 us, in pairs 261).
template <int kForm>
constexpr bool few_pairs(int depth)
{
    return FewForm<kForm>::kQ4 && depth >= 4;
}

// First line of part `part` of `parts` of a reduction (of part `parts`: its end).  Pairs are in one part.
template <int kForm>
__device__ __forceinline__ int few_part_line(int lines, int part, int parts)
{
    if constexpr (!FewForm<kForm>::kQ4)
        return lines * part / parts;
    const int line = (lines + 1) / 2 * part / parts * 2;
    return line < lines ? line : lines;
}

// A wavefront's stream: segment after segment (a panel of weight rows with the activation rows that meet it, some lines of
// both), without a gap in the loads between them.  The source says what they are:
//   open(cursor)    sets the cursor to the next segment, with at least one group of kDepth lines (lines past its end read as
//                   zeros); false: there is none.  A group ahead of
//   close(sums)     takes the sums of the oldest open segment
// A group is written out straight, so that what is waited for is the same on every path: segments change between groups only.
// (With a change possible at every line the code is kDepth times as long, 180 KB, and waits for nearly everything in flight.)
template <int kForm, int kTT, int kCT, int kDepth, int kActs, class Source>
__device__ __forceinline__ void few_stream(Source &source, const FewCols &g)
{
    using Form = FewForm<kForm>;
    using Ops = FewOperands<kForm, kTT, kCT>;
    using Cursor = FewCursor<kForm, kTT, kCT, kActs>;
    Cursor c;
    if (!source.open(c))
        return;
    const int i = threadIdx.x % kWave / 4, q = threadIdx.x % 4; // whose operand this lane fetches
    constexpr bool kPairs = few_pairs<kForm>(kDepth);
    const uint32_t row_bytes = (uint32_t)Form::row_bytes(g.cols);
    const uint32_t w_off = kPairs ? (uint32_t)(i % 8) * row_bytes + (uint32_t)(i / 8 * 64 + q * 16) : (uint32_t)i * row_bytes + (uint32_t)q * 16u;
    constexpr int kFours = Form::kQ4 ? (kDepth + 3) / 4 : 1; // scale loads per group of lines
    FewScales<kForm, kCT> scales[kFours];
    auto fetch = [&](Ops &o, int d) {
        const int odd = kPairs ? d % 2 : 0;
        const bool there = c.line < c.end, w_there = c.line - odd < c.end; // (else no bytes: zeros, and the number of loads in flight stays)
#pragma unroll
        for (int p = 0; p < kCT; ++p) {
            const auto rw = few_buffer(c.panel[p].data, w_there ? c.panel[p].bytes : 0u);
#pragma unroll
            for (int s = 0; s < Form::kLoads; ++s) {
                uint32_t at = w_off + (uint32_t)((c.line - odd) * Form::kLineBytes + 64 * s) + (odd ? 8 * row_bytes : 0u);
                if constexpr (kForm == kFewF32) // (past the row's end: the next row's, whose infinities and NaN stay its own)
                    at |= c.line * Form::kLineCols + 16 * s + 4 * q < g.cols ? 0u : kNowhere;
                o.w[p][s] = __builtin_amdgcn_raw_buffer_load_b128(rw, (int)at, 0, 0);
            }
        }
        const auto ra = few_buffer(c.act, there ? c.act_bytes : 0u);
#pragma unroll
        for (int t = 0; t < Ops::kActs; ++t) {
            const int col = c.line * Form::kLineCols + Cursor::lane_col(t);
            // (past the row's end would be another row's)
            const uint32_t at = c.col_off(col) | (!Form::kRagged || kActs == kActPacked || col < g.cols ? 0u : kNowhere);
#pragma unroll
            for (int m = 0; m < Ops::kRows; ++m)
                o.a[m][t] = __builtin_amdgcn_raw_buffer_load_b128(ra, (int)(at + c.row_off[m]), 0, 0);
        }
        ++c.line;
        // one order of the loads everywhere: else the wait at the top of the loop is for all of them
        __builtin_amdgcn_sched_barrier(0);
    };
    // the scales of a group of lines, asked for before its first line
    auto fetch_scales = [&]() {
        if constexpr (Form::kQ4) {
            constexpr int kBytes = kForm == kFewFp4 ? 1 : 2, kLoad = 4 * FewScales<kForm, kCT>::kRegs;
            constexpr int per_line = 4 / Form::kSame;
            const int groups = g.scale_cols < c.end * per_line ? g.scale_cols : c.end * per_line;
#pragma unroll
            for (int f = 0; f < kFours; ++f) {
                const int left = groups - (c.line + 4 * f + q) * per_line;
#pragma unroll
                for (int r = 0; r < FewScales<kForm, kCT>::kRegs; ++r) {
                    constexpr int per_reg = 4 / kBytes;
                    const int n = left - per_reg * r;
                    scales[f].keep[r] = n >= per_reg ? 0xFFFFFFFFu : n > 0 ? (1u << (8 * kBytes * n)) - 1 : 0u;
                }
#pragma unroll
                for (int p = 0; p < kCT; ++p) {
                    const auto rs = few_buffer(c.panel[p].scales, c.line < c.end ? c.panel[p].scale_bytes : 0u);
                    const uint32_t want = (uint32_t)(i * g.scale_cols + (c.line + 4 * f + q) * per_line) * kBytes;
                    const uint32_t last = c.panel[p].scale_bytes - kLoad, at = want < last ? want : last;
                    scales[f].shift[p] = want - at < kLoad ? 8 * (want - at) : 0; // (further: of a row or line that is not there)
                    if constexpr (kLoad == 4) {
                        scales[f].raw[p][0] = __builtin_amdgcn_raw_buffer_load_b32(rs, (int)at, 0, 0);
                    } else {
                        const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(rs, (int)at, 0, 0);
                        scales[f].raw[p][0] = v[0], scales[f].raw[p][1] = v[1];
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    Ops o[kDepth];
    int left = c.groups, next = 0; // groups of the segment that is multiplied, and of the one after it (0: there is none)
    fetch_scales();
#pragma unroll
    for (int d = 0; d < kDepth; ++d)
        fetch(o[d], d);
    FewSums<kForm, kTT, kCT> sums;
    sums.clear();
    if constexpr (kPairs)
        few_to_lines(o[0], o[1]);
    to_operand_lanes<kForm, kTT, kCT, kActs>(o[0]);
    for (;;) {
        if (--c.groups == 0) { // the next group is another segment's
            if (source.open(c)) {
                next = c.groups;
            } else {
                next = 0;
                c.end = 0; // nothing more: no bytes
            }
        }
        if constexpr (Form::kQ4) {
#pragma unroll
            for (int f = 0; f < kFours; ++f)
                scales[f].template spread<(kActs != kActRows && Form::kOwn)>();
            __builtin_amdgcn_sched_barrier(0);
        }
        fetch_scales();
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            // (a line changes lanes under the products of the one before)
            const int next = (d + 1) % kDepth;
            if constexpr (kPairs)
                if (next % 2 == 0)
                    few_to_lines(o[next], o[next + 1]);
            to_operand_lanes<kForm, kTT, kCT, kActs>(o[next]);
            __builtin_amdgcn_sched_barrier(0);
            few_multiply<kForm, kTT, kCT, kActs>(sums, o[d], scales[Form::kQ4 ? d / 4 : 0], d % 4);
            __builtin_amdgcn_sched_barrier(0);
            fetch(o[d], d);
        }
        if (--left == 0) {
            source.close(sums);
            if (next == 0)
                return;
            sums.clear();
            left = next;
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

// The wavefronts of a workgroup draw units: items, or one of `parts` parts of an item's reduction.

// The next number of a counter in LDS, for the wavefront.
__device__ __forceinline__ int few_draw(int *counter)
{
    int n = 0;
    if (threadIdx.x % kWave == 0)
        n = atomicAdd(counter, 1);
    return __builtin_amdgcn_readfirstlane(n);
}

// Parts (1, 2, 4 or 8) with which a workgroup's wavefronts are soonest through `items` items of `lines` lines each: a unit
// takes whole groups of `depth` lines, and some time of its own; parts also meet in LDS.
__device__ __forceinline__ int few_parts(int items, int lines, int depth)
{
    int best = 1, least = 0x7FFFFFFF;
    for (int parts = 1; parts <= kFewWaves && (parts == 1 || parts <= lines); parts *= 2) {
        const int turns = (items * parts + kFewWaves - 1) / kFewWaves, length = (lines + parts - 1) / parts;
        const int time = turns * ((length + depth - 1) / depth * depth + (parts > 1 ? 3 : 2));
        if (time < least)
            least = time, best = parts;
    }
    return best;
}

// Room in LDS for items whose parts are under way: how far wavefronts may be apart.
struct FewRoom {
    int parts_done[8]; // of the item in a place
    int item[8];       // that may use a place
};

// Where the parts of items 0, 1, .. of a workgroup meet.  A place in the pool is [part][tile][value][lane].
template <int kForm, int kTT, int kCT>
struct FewJoin {
    static constexpr int kValues = kFewValues<kForm, kTT>, kPartFloats = kCT * kValues * kWave;
    float *pool;
    FewRoom &room;
    int parts, places;

    __device__ FewJoin(float *pool, int pool_floats, FewRoom &room, int parts) : pool(pool), room(room), parts(parts)
    {
        places = pool_floats / (parts * kPartFloats);
        places = places < 8 ? places : 8;
    }
    // Part `part` of item n; whoever brings the last one calls done(total) with total(tile, value), added up in the parts'
    // order.  A part waits until the item that had its place before is done with.  The oldest item that is not done never
    // waits, and every wavefront closes its units in the order of their items: so every wait ends.
    template <class Done>
    __device__ __forceinline__ void close(const FewSums<kForm, kTT, kCT> &sums, int n, int part, Done done)
    {
        const int lane = threadIdx.x % kWave, place = n % places;
        while (__builtin_amdgcn_readfirstlane(__hip_atomic_load(&room.item[place], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)) != n)
            __builtin_amdgcn_s_sleep(1);
        float *const slot = pool + place * parts * kPartFloats;
#pragma unroll
        for (int c = 0; c < kCT; ++c)
#pragma unroll
            for (int v = 0; v < kValues; ++v)
                slot[part * kPartFloats + (c * kValues + v) * kWave + lane] = sums.value(c, v);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // (LDS of a workgroup keeps its order)
        if (few_draw(&room.parts_done[place]) != parts - 1)
            return;
        asm volatile("" ::: "memory");
        done([&](int c, int v) {
            float p[kFewWaves];
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) // (past the last part: the first, for nothing)
                p[w] = slot[(w < parts ? w : 0) * kPartFloats + (c * kValues + v) * kWave + lane];
            float all = p[0];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w)
                all += w < parts ? p[w] : 0.0f;
            return all;
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (lane == 0) {
            room.parts_done[place] = 0;
            asm volatile("" ::: "memory"); // (before the place is given away)
            __hip_atomic_store(&room.item[place], n + places, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        }
    }
};
#endif

}  // namespace moe

// The whole layer for a few tokens: router logits and the launches (few_ffn.h has the rest of the layer).
#include <math.h>

#include <atomic>

#include "common.h"
#include "few.h"
#include "few_ffn.h"

namespace moe {

// Logits in moe_route's order (route.hip, "R64"): partial l of 64 takes h = l, l + 64, ... by single fused multiply-adds,
// which v_mfma_f32_16x16x1_4B_f32 does for four partials of 16 tokens x 16 experts at a time; then rounds 32, 16, ... 1.
// A workgroup has sixteen experts and the eight partials l = j, j + 8, ... (wavefront 0: the first four), which rounds 32,
// 16 and 8 make one; the reader does rounds 4, 2, 1.  So even one token's router runs on E / 2 workgroups, and an XCD
// (j = blockIdx.x % 8) has rows of W_r of its own.  Latency bound: all loads of 64 steps are in flight at once.
// Further workgroups write x as the products with 4-bit weights want it (few_stream.h): a line's sixteens of eight columns
// in the order of FewForm::kOwn (`own`), the columns of eight in int4_order (`order`), zeros past H.
// ------------------------------------------------------------------------
template <bool kBf16>
__global__ __launch_bounds__(2 * kWave) void few_logits(const void *__restrict__ x, int N, int H, const float *__restrict__ W_r,
                                                        int E, float *__restrict__ parts, uint32_t *flags, int flag_count, u32x4 *packed, int own,
                                                        int order)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kBatch = 32;
    __shared__ float fold[16 * kWave];
    const int lane = threadIdx.x % kWave, c = lane % 16, blk = lane / 16;
    const int half = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int j = (int)blockIdx.x % kParts, e0 = (int)blockIdx.x / kParts * 16, n0 = (int)blockIdx.y * 16;
    const int logit_groups = (E + 15) / 16 * kParts;
    if ((int)blockIdx.x >= logit_groups) {
        if constexpr (kBf16) {
            const int row = (H + 127) / 128 * 16, at = (((int)blockIdx.x - logit_groups) * (int)gridDim.y + (int)blockIdx.y) * (2 * kWave) + (int)threadIdx.x;
            const int n = at / row, u = at % row;
            if (n < N) {
                u32x4 v = {0, 0, 0, 0};
                if (8 * u < H)
                    v = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(x) + (int64_t)n * H + 8 * u);
                packed[n * row + (own ? u / 16 * 16 + u % 4 * 4 + u / 4 % 4 : u)] = order ? __builtin_bit_cast(u32x4, int4_order(v)) : v;
            }
        }
        return;
    }
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (int f = threadIdx.x; f < flag_count; f += 2 * kWave)
            flags[f] = 0;
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

struct FewWorkspace {
    uint32_t *flags;
    float *parts;
    void *x; // packed
    void *a;
    size_t bytes;
};

static FewWorkspace few_carve(void *ws, int64_t N, int64_t H, int E, int K, int64_t F, int dtype)
{
    unsigned char *const w = static_cast<unsigned char *>(ws);
    const size_t elt = dtype == MOE_BF16 ? 2 : 4;
    const size_t parts = kFlags * sizeof(uint32_t), x = parts + ((size_t)N * kParts * E * sizeof(float) + 127) / 128 * 128;
    const size_t a = x + (dtype == MOE_BF16 ? (size_t)N * ((H + 127) / 128) * 256 : 0);
    // tiles of at least 8 columns, each expert's (an expert may have two entries) in whole cache lines: at most 15 bytes a
    // column are lost
    const size_t rows = (size_t)N * K, experts = (rows < (size_t)E ? rows : (size_t)E) + rows / (kFewMost + 1), cols = F + 32;
    return {reinterpret_cast<uint32_t *>(w), reinterpret_cast<float *>(w + parts), w + x, w + a,
            a + rows * cols * elt + experts * cols * 16};
}

size_t few_workspace_bytes(int64_t N, int64_t H, int E, int K, int64_t F, int dtype)
{
    return few_carve(nullptr, N, H, E, K, F, dtype).bytes;
}

// Width of the gate/up items: the least time of the longest share, in units of a line of one column per wavefront, with the
// parts that few_parts will choose about like here.  Narrow items make even shares of little work (one token, 4 experts of
// 1408 columns: 22 columns per workgroup, three items of 8 or two of 16: 26.3 and 27.0 us for the second launch), wide ones use
// their loads better (37 tokens of 32 experts fp4: 194 and 169 us), and in single precision the matrix instructions, half of
// which 8 columns leave empty (5 tokens of 12 experts: 49 and 47 us), are the bound.
static int choose_width(const FewKernelArgs &g, double experts, int narrowest)
{
    int64_t least = INT64_MAX;
    int best = 16;
    for (int width = 16; width >= narrowest; width /= 2)
        for (int parts = 1; parts <= kFewWaves && (parts == 1 || parts <= g.h_lines); parts *= 2) {
            const int64_t items = ceil_div((int64_t)(experts * (double)ceil_div(g.l.F, width) + 0.5), g.shares);
            const int64_t turns = ceil_div(items * parts, kFewWaves);
            const int64_t time = turns * (ceil_div(ceil_div(g.h_lines, parts), 4) * 4 * (width + 4) + (parts > 1 ? 12 : 8));
            if (time < least)
                least = time, best = width;
        }
    return best;
}

// Polls (about a microsecond each) that a workgroup waits for others' shares: 60, and what the largest share's weights take at
// 8 GB/s, a third of a compute unit's part of the memory's rate.  That is longer than any share takes with the card to itself (the
// layers alone take the same time with 30 and with 250) and shorter than much more work would be: one token of 4 experts on four
// streams at once, 282 us for the four with 250, 192 with 60, 177 with 30; one after the other 139.
static int choose_patience(const FewKernelArgs &g, double experts, int64_t row_bytes)
{
    const double items = ceil(experts * (double)g.f_tiles / g.shares);
    return (int)fmin(60.0 + items * 2.0 * g.width * (double)row_bytes / 8e3, 1e6);
}

static std::atomic<int> test_polls{-1}, test_workgroups{0};
extern "C" void moe_few_test_waits(int polls, int workgroups)
{
    test_polls.store(polls, std::memory_order_relaxed);
    test_workgroups.store(workgroups, std::memory_order_relaxed);
}

int launch_layer_few(const FewArgs &args, int dtype, int format, hipStream_t st)
{
    const FewWorkspace w = few_carve(args.ws, args.N, args.H, args.E, args.K, args.F, dtype);
    const int cus = compute_units();
    FewKernelArgs g = {};
    g.l = args;
    g.l.a = w.a;
    g.parts = w.parts;
    g.flags = w.flags;
    g.shares = cus < kMaxShares ? cus : kMaxShares;
    const int line_cols = format != kNoFormat ? 128 : dtype == MOE_BF16 ? 64 : 32;
    g.h_lines = (int)ceil_div(args.H, line_cols);
    g.f_lines = (int)ceil_div(args.F, line_cols);
    const int rows = args.N * args.K;
    const double touched = args.E * (1.0 - pow(1.0 - (double)args.K / args.E, args.N)); // experts, if all are equally popular
    const double experts = touched < 1.0 ? 1.0 : touched;
    g.width = choose_width(g, experts, dtype == MOE_BF16 ? 8 : 16);
    g.f_tiles = (int)ceil_div(args.F, g.width);
    // columns of a down tile: as many tiles as workgroups (or a multiple), none wider than 32, or 16 where the rows' sums would
    // not fit in LDS
    const int64_t widest = rows * 32 <= kPoolFloats ? 32 : 16, rounds = ceil_div(args.H, widest * g.shares);
    g.down_cols = (int)(ceil_div(ceil_div(args.H, rounds * g.shares), 4) * 4);
    // parts of an expert there: some eight units for each wavefront, none shorter than eight lines (a ring of the fewest rows)
    const int row_floats = g.down_cols <= 16 ? 16 : 32;
    for (g.down_parts = 1; g.down_parts < 16 && experts * g.down_parts < 8 * kFewWaves && g.f_lines >= 16 * g.down_parts &&
                           2 * g.down_parts * rows * row_floats <= kPoolFloats;)
        g.down_parts *= 2;
    const int polls = test_polls.load(std::memory_order_relaxed);
    const int64_t row_bytes = format != kNoFormat ? args.H / 2 : (int64_t)args.H * (dtype == MOE_BF16 ? 2 : 4);
    g.patience = polls < 0 ? choose_patience(g, rows < args.E ? rows : args.E, row_bytes) : polls;
    const int workgroups = test_workgroups.load(std::memory_order_relaxed);
    g.workgroups = workgroups > 0 && workgroups < g.shares ? workgroups : g.shares;
    const bool packed = format != kNoFormat;
    g.x = packed ? w.x : args.x;
    g.x_cols = packed ? g.h_lines * 128 : args.H;
    const int64_t rows16 = ceil_div(args.N, 16), copies = packed ? ceil_div((int64_t)args.N * g.h_lines * 16, 2 * kWave * rows16) : 0;
    const dim3 grid((unsigned)(ceil_div(args.E, 16) * kParts + copies), (unsigned)rows16);
    const int own = format == MOE_Q4_FP4 || args.group == 128, order = format == MOE_Q4_INT4;
    if (dtype == MOE_BF16)
        hipLaunchKernelGGL(few_logits<true>, grid, dim3(2 * kWave), 0, st, args.x, args.N, args.H, args.W_r, args.E, w.parts, w.flags, kFlags,
                           static_cast<u32x4 *>(w.x), own, order);
    else
        hipLaunchKernelGGL(few_logits<false>, grid, dim3(2 * kWave), 0, st, args.x, args.N, args.H, args.W_r, args.E, w.parts, w.flags, kFlags,
                           static_cast<u32x4 *>(w.x), own, order);
    if (format == MOE_Q4_FP4)
        launch_few_ffn<kFewFp4>(g, st);
    else if (format == MOE_Q4_INT4 && args.group == 32)
        launch_few_ffn<kFewInt4By32>(g, st);
    else if (format == MOE_Q4_INT4 && args.group == 64)
        launch_few_ffn<kFewInt4By64>(g, st);
    else if (format == MOE_Q4_INT4)
        launch_few_ffn<kFewInt4By128>(g, st);
    else if (dtype == MOE_BF16)
        launch_few_ffn<kFewBf16>(g, st);
    else
        launch_few_ffn<kFewF32>(g, st);
    return check_launch("moe_layer_few");
}

}  // namespace moe

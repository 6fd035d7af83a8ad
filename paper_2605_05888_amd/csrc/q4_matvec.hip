// Products of a few rows with 4-bit matrices: few_stream.h's stream, one panel of weight rows per workgroup.
#include "common.h"
#include "few.h"
#include "few_stream.h"

namespace moe {

constexpr int kMvWaves = 8;

#if defined(__HIP_DEVICE_COMPILE__)
// Rows [m0, m0 + rows) of x, at most 16 kTT (kTT = 0: 4), with weight rows [n0, n0 + 16 kCT) of matrix e.
template <int kForm, int kTT, int kCT, int kDepth>
struct MatvecTile {
    using Form = FewForm<kForm>;
    const MatvecArgs &g;
    float *red;
    int e;
    int64_t m0;
    int rows;
    int64_t n0;
    bool opened = false;

    __device__ __forceinline__ int lines() const { return (g.cols + Form::kLineCols - 1) / Form::kLineCols; }
    __device__ __forceinline__ int wave() const { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); }
    __device__ __forceinline__ int first() const { return lines() * wave() / kMvWaves; }
    __device__ __forceinline__ int last() const { return lines() * (wave() + 1) / kMvWaves; }
    __device__ __forceinline__ bool open(FewCursor<kForm, kTT, kCT, false> &c)
    {
        if (opened)
            return false;
        opened = true;
        const int64_t row = (int64_t)e * g.rows + n0, end = (int64_t)(e + 1) * g.rows;
#pragma unroll
        for (int p = 0; p < kCT; ++p)
            c.panel[p] = panel_of<kForm>(g.w, row + 16 * p, end, g.cols, g.scale_cols);
        const uint32_t x_row = (uint32_t)g.cols * Form::kElt;
        c.set_acts({static_cast<const unsigned char *>(g.x) + m0 * x_row, (uint32_t)rows * x_row, 0, 0, rows},
                   [&](int r) { return r * x_row; });
        c.line = first();
        c.end = last();
        c.groups = last() > first() ? (last() - first() + kDepth - 1) / kDepth : 1;
        return true;
    }
    __device__ __forceinline__ void close(const FewSums<kForm, kTT, kCT> &sums) const
    {
        constexpr int kValues = kFewValues<kForm, kTT>;
        const int lane = threadIdx.x % kWave;
#pragma unroll
        for (int c = 0; c < kCT; ++c)
#pragma unroll
            for (int v = 0; v < kValues; ++v)
                red[((wave() * kCT + c) * kValues + v) * kWave + lane] = sums.value(c, v);
        few_barrier();
        for (int o = wave(); o < kCT * kValues; o += kMvWaves) {
            float v = red[o * kWave + lane];
#pragma unroll
            for (int w = 1; w < kMvWaves; ++w)
                v += red[(w * kCT * kValues + o) * kWave + lane];
            const int r = few_row_of<kForm, kTT>(o % kValues);
            const int64_t n = n0 + 16 * (o / kValues) + lane % 16;
            const uint32_t both = pack_bf16x2(v, __shfl_xor(v, 1)); // the even lane stores both columns
            if (r < rows && n < g.rows && lane % 2 == 0)
                *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(g.y) + (m0 + r) * g.rows + n) = both;
        }
        few_barrier(); // (red is written again by the next rows)
    }
};
#endif

template <int kForm, int kMaxTT, int kCT>
__global__ __launch_bounds__(kMvWaves *kWave, kMaxTT == 1 ? 4 : 2) void q4_matvec(MatvecArgs g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ float red[kMvWaves * kCT * 4 * kMaxTT * kWave];
    const int e = (int)blockIdx.y;
    const int64_t n0 = (int64_t)blockIdx.x * 16 * kCT;
    const int64_t m1 = g.seg_offsets ? g.seg_offsets[e + 1] : g.M;
    for (int64_t m0 = g.seg_offsets ? g.seg_offsets[e] : 0; m0 < m1; m0 += 16 * kMaxTT) {
        const int rows = (int)(m1 - m0 < 16 * kMaxTT ? m1 - m0 : 16 * kMaxTT);
        const FewCols cols = {g.cols, g.scale_cols, g.group};
        auto tile = [&](auto tt, auto depth) {
            constexpr int kTT = decltype(tt)::value, kDepth = decltype(depth)::value;
            MatvecTile<kForm, kTT, kCT, kDepth> t = {g, red, e, m0, rows, n0};
            few_stream<kForm, kTT, kCT, kDepth, false>(t, cols);
        };
        if (rows <= FewForm<kForm>::kFewRows)
            tile(std::integral_constant<int, 0>{}, std::integral_constant<int, 4>{});
        else if (kMaxTT == 1 || rows <= 16)
            tile(std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
        else if (rows <= 32)
            tile(std::integral_constant<int, (kMaxTT < 2 ? 1 : 2)>{}, std::integral_constant<int, 4>{});
        else
            tile(std::integral_constant<int, kMaxTT>{}, std::integral_constant<int, 2>{});
    }
#endif
}

template <int kForm>
static void launch(const MatvecArgs &g, int E_local, hipStream_t st)
{
    const dim3 block(kMvWaves * kWave);
    if (g.M <= 16)
        hipLaunchKernelGGL((q4_matvec<kForm, 1, 1>), dim3((unsigned)ceil_div(g.rows, 16), (unsigned)E_local), block, 0, st, g);
    else
        hipLaunchKernelGGL((q4_matvec<kForm, 4, 2>), dim3((unsigned)ceil_div(g.rows, 32), (unsigned)E_local), block, 0, st, g);
}

int launch_matvec_q4(const MatvecArgs &g, int E_local, int format, hipStream_t st)
{
    if (format == MOE_Q4_FP4)
        launch<kFewFp4>(g, E_local, st);
    else
        launch<kFewInt4>(g, E_local, st);
    return check_launch("moe_matvec_q4");
}

}  // namespace moe

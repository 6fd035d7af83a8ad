// The decoding operators: a whole layer for a few tokens, and products of a few rows with 4-bit matrices.
// Simple form: a wavefront computes one element of a product.
#include <math.h>

#include "common.h"
#include "few.h"
#include "q4.h"

namespace moe {

constexpr int kFewThreads = 256, kFewWaves = kFewThreads / kWave;

// How a weight matrix is held; activations are bf16 but for kF32.
enum { kFewBf16 = 0, kFewF32 = 1, kFewFp4 = 2, kFewInt4 = 3 };

#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1)
        v += __shfl_xor(v, s);
    return v;
}

template <int kForm>
__device__ __forceinline__ float act_value(const void *x, int64_t at)
{
    if constexpr (kForm == kFewF32)
        return static_cast<const float *>(x)[at];
    else
        return bf16_bits_to_f32(static_cast<const uint16_t *>(x)[at]);
}

// sum over columns of W[row, c] x[at + c], the whole wavefront
template <int kForm>
__device__ __forceinline__ float row_dot(const FewMatrix &w, int64_t row, int cols, int group, int scale_cols, const void *x,
                                         int64_t at)
{
    const int lane = threadIdx.x % kWave;
    float sum = 0.0f;
    if constexpr (kForm == kFewBf16 || kForm == kFewF32) {
        for (int c = lane; c < cols; c += kWave)
            sum = fmaf(act_value<kForm>(w.data, row * cols + c), act_value<kForm>(x, at + c), sum);
    } else {
        for (int c = lane * 8; c < cols; c += kWave * 8) {
            const uint32_t codes = static_cast<const uint32_t *>(w.data)[(row * cols + c) / 8];
            float v[8];
            const int64_t s = row * scale_cols + c / group;
            if constexpr (kForm == kFewFp4)
                q4_values<MOE_Q4_FP4>(codes, fp4_scale(static_cast<const unsigned char *>(w.scales)[s]), v);
            else
                q4_values<MOE_Q4_INT4>(codes, bf16_bits_to_f32(static_cast<const uint16_t *>(w.scales)[s]), v);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                sum = fmaf(v[j], act_value<kForm>(x, at + c + j), sum);
        }
    }
    return wave_sum(sum);
}

template <int kForm>
__device__ __forceinline__ void put(void *y, int64_t at, float v)
{
    if constexpr (kForm == kFewF32)
        static_cast<float *>(y)[at] = v;
    else
        static_cast<uint16_t *>(y)[at] = (uint16_t)f32_to_bf16_bits(v);
}
#endif

// element (row r = n * K + k, column f) of the activation
template <int kForm>
__global__ __launch_bounds__(kFewThreads) void few_gate_up(FewArgs g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const int64_t f = (int64_t)blockIdx.x * kFewWaves + threadIdx.x / kWave;
    const int r = (int)blockIdx.y;
    if (f >= g.F)
        return;
    const int64_t row = (int64_t)g.topk_idx[r] * g.F + f, at = (int64_t)(r / g.K) * g.H;
    const float gate = row_dot<kForm>(g.gate, row, g.H, g.group, g.scale_cols_h, g.x, at);
    const float up = row_dot<kForm>(g.up, row, g.H, g.group, g.scale_cols_h, g.x, at);
    if (threadIdx.x % kWave == 0)
        put<kForm>(g.a, (int64_t)r * g.F + f, gate / (1.0f + expf(-gate)) * up);
#endif
}

template <int kForm>
__global__ __launch_bounds__(kFewThreads) void few_down(FewArgs g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const int64_t h = (int64_t)blockIdx.x * kFewWaves + threadIdx.x / kWave;
    const int n = (int)blockIdx.y;
    if (h >= g.H)
        return;
    float sum = 0.0f;
    for (int k = 0; k < g.K; ++k) {
        const int r = n * g.K + k;
        sum += g.topk_w[r] *
               row_dot<kForm>(g.down, (int64_t)g.topk_idx[r] * g.H + h, g.F, g.group, g.scale_cols_f, g.a, (int64_t)r * g.F);
    }
    if (threadIdx.x % kWave == 0)
        put<kForm>(g.out, (int64_t)n * g.H + h, sum);
#endif
}

template <int kForm>
__global__ __launch_bounds__(kFewThreads) void matvec(MatvecArgs g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const int64_t n = (int64_t)blockIdx.x * kFewWaves + threadIdx.x / kWave;
    const int e = (int)blockIdx.y;
    if (n >= g.rows)
        return;
    const int64_t m0 = g.seg_offsets ? g.seg_offsets[e] : 0, m1 = g.seg_offsets ? g.seg_offsets[e + 1] : g.M;
    for (int64_t m = m0; m < m1; ++m) {
        const float v = row_dot<kForm>(g.w, (int64_t)e * g.rows + n, g.cols, g.group, g.scale_cols, g.x, m * g.cols);
        if (threadIdx.x % kWave == 0)
            put<kForm>(g.y, m * g.rows + n, v);
    }
#endif
}

size_t few_workspace_bytes(int64_t N, int64_t H, int E, int K, int64_t F, int dtype)
{
    (void)H;
    const size_t logits = ((size_t)N * (size_t)E * sizeof(float) + 127) / 128 * 128;
    return logits + (size_t)N * (size_t)K * (size_t)F * (dtype == MOE_BF16 ? 2 : 4) + 128;
}

template <int kForm>
static void launch_layer(const FewArgs &g, hipStream_t st)
{
    hipLaunchKernelGGL(few_gate_up<kForm>, dim3((unsigned)ceil_div(g.F, kFewWaves), (unsigned)(g.N * g.K)), dim3(kFewThreads), 0,
                       st, g);
    hipLaunchKernelGGL(few_down<kForm>, dim3((unsigned)ceil_div(g.H, kFewWaves), (unsigned)g.N), dim3(kFewThreads), 0, st, g);
}

int launch_layer_few(const FewArgs &args, int dtype, int format, hipStream_t st)
{
    FewArgs g = args;
    float *const logits = static_cast<float *>(g.ws);
    g.a = static_cast<unsigned char *>(g.ws) + ((size_t)g.N * g.E * sizeof(float) + 127) / 128 * 128;
    const int rc = launch_route(g.x, dtype, g.N, g.H, g.W_r, g.bias, g.E, g.K, g.score_mode, g.topk_idx, g.topk_w, logits, st);
    if (rc != MOE_OK)
        return rc;
    if (format == MOE_Q4_FP4)
        launch_layer<kFewFp4>(g, st);
    else if (format == MOE_Q4_INT4)
        launch_layer<kFewInt4>(g, st);
    else if (dtype == MOE_BF16)
        launch_layer<kFewBf16>(g, st);
    else
        launch_layer<kFewF32>(g, st);
    return check_launch("moe_layer_few");
}

int launch_matvec_q4(const MatvecArgs &g, int E_local, int format, hipStream_t st)
{
    const dim3 grid((unsigned)ceil_div(g.rows, kFewWaves), (unsigned)E_local);
    if (format == MOE_Q4_FP4)
        hipLaunchKernelGGL(matvec<kFewFp4>, grid, dim3(kFewThreads), 0, st, g);
    else
        hipLaunchKernelGGL(matvec<kFewInt4>, grid, dim3(kFewThreads), 0, st, g);
    return check_launch("moe_matvec_q4");
}

}  // namespace moe

// 4-bit weights: a matrix into codes and scales, and back.
//
// Both are one pass over memory: 2 or 4 bytes a weight on one side, 0.53 on the other.  FP4 and the way back are bound by it
// (14336 x 4096 bf16: 33 and 23 us, 79 - 109 instructions for eight weights); to INT4 it is 441 instructions, the exact quotient and
// its borders, and these are the bound (85 us).  A lane takes eight columns (16 or 32 bytes of W, one register of codes), so that a
// wavefront's accesses are contiguous on either side, and kPer such units far apart, whose loads are all in flight
// before the first is used.  The lanes of a group stand side by side: its largest magnitude is a few lane exchanges.
#include <math.h>

#include "common.h"
#include "q4.h"

namespace moe {

constexpr int kQ4Threads = 256, kQ4Per = 4;

struct Q4Args {
    const void *w_in;
    void *w_out;
    unsigned char *codes, *scales;
    int64_t rows;
    int cols, group, scale_cols;
    int units; // eight columns each, per row; rounded up to whole groups, so that a group never crosses a wavefront
};

// Unit p of the rounded-up grid of units: its row and first column (col >= cols: not there).
struct Q4Unit {
    int64_t row;
    int col;
};

#if defined(__HIP_DEVICE_COMPILE__)
// Units of a workgroup lie side by side: one 64-bit division for all, 32-bit ones for the lanes.
struct Q4Walk {
    int64_t row0;
    uint32_t rest, units;
    __device__ Q4Walk(const Q4Args &g)
    {
        const int64_t first = (int64_t)blockIdx.x * (kQ4Threads * kQ4Per);
        units = (uint32_t)g.units;
        row0 = first / units;
        rest = (uint32_t)(first - row0 * units);
    }
    __device__ Q4Unit at(int i) const
    {
        const uint32_t p = rest + (uint32_t)(i * kQ4Threads) + threadIdx.x, r = p / units;
        return {row0 + r, (int)((p - r * units) * 8u)};
    }
};

struct Eight {
    float v[8];
};
template <bool kBf16>
__device__ __forceinline__ Eight load_eight(const void *w, int64_t at)
{
    Eight e;
    if constexpr (kBf16) {
        const u32x4 r = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(w) + at));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            e.v[2 * i] = __uint_as_float(r[i] << 16), e.v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
    } else {
        const f32x4 *p = reinterpret_cast<const f32x4 *>(static_cast<const float *>(w) + at);
        const f32x4 a = __builtin_nontemporal_load(p), b = __builtin_nontemporal_load(p + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            e.v[i] = a[i], e.v[4 + i] = b[i];
    }
    return e;
}

// m / 7 rounded once to bf16.  The fp32 quotient is within half a unit of its last place; only where it lands on a
// border between two bf16 numbers the remainder m - 7 q, exact by one fused multiply-add, says which side m / 7 is on.
__device__ __forceinline__ uint32_t int4_scale_bits(float m)
{
    const float q = m / 7.0f;
    const uint32_t b = __float_as_uint(q);
    uint32_t up = 0x7FFFu + ((b >> 16) & 1u);
    if ((b & 0xFFFFu) == 0x8000u) {
        const float r = fmaf(-7.0f, q, m);
        up = r > 0.0f ? 0x8000u : r < 0.0f ? 0x7FFFu : up;
    }
    return (b + up) >> 16;
}

// w / s to the nearest whole number, ties to even, within -8 .. 7, from the exact quotient: the borders (k + 1/2) s are
// exact in fp32 (s has 8 bits), so the rounded quotient's whole number is put right by comparing with them.
__device__ __forceinline__ int int4_code(float w, float s)
{
    const float a = fabsf(w);
    float k = fminf(rintf(a / s), 8.0f);
    const float low = (k - 0.5f) * s, high = (k + 0.5f) * s;
    const bool odd = ((int)k & 1) != 0;
    if (a < low || (a == low && odd))
        k -= 1.0f;
    else if (a > high || (a == high && odd))
        k += 1.0f;
    return w < 0.0f ? 8 - (int)fminf(k, 8.0f) : 8 + (int)fminf(k, 7.0f);
}
#endif

template <int kFormat, bool kBf16>
__global__ __launch_bounds__(kQ4Threads) void q4_quantize(Q4Args g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const Q4Walk walk(g);
    Eight e[kQ4Per];
    Q4Unit u[kQ4Per];
#pragma unroll
    for (int i = 0; i < kQ4Per; ++i) {
        u[i] = walk.at(i);
        if (u[i].row < g.rows && u[i].col < g.cols)
            e[i] = load_eight<kBf16>(g.w_in, u[i].row * g.cols + u[i].col);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j)
                e[i].v[j] = 0.0f;
    }
    const int lanes = g.group / 8; // of a group: 4, 8 or 16
#pragma unroll
    for (int i = 0; i < kQ4Per; ++i) {
        float m = fabsf(e[i].v[0]);
#pragma unroll
        for (int j = 1; j < 8; ++j)
            m = fmaxf(m, fabsf(e[i].v[j]));
        m = fmaxf(m, __shfl_xor(m, 1));
        m = fmaxf(m, __shfl_xor(m, 2));
        if (kFormat == MOE_Q4_INT4) {
            if (lanes >= 8)
                m = fmaxf(m, __shfl_xor(m, 4));
            if (lanes >= 16)
                m = fmaxf(m, __shfl_xor(m, 8));
        }
        if (!(u[i].row < g.rows && u[i].col < g.cols))
            continue;
        uint32_t code = 0, scale_bits;
        if constexpr (kFormat == MOE_Q4_FP4) {
            const int s = (int)(__float_as_uint(m) >> 23) - 2;
            scale_bits = s < 1 ? 1u : (uint32_t)s;
            const float scale = fp4_scale(scale_bits);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, e[i].v[0], e[i].v[1], scale, 0);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, e[i].v[2], e[i].v[3], scale, 1);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, e[i].v[4], e[i].v[5], scale, 2);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, e[i].v[6], e[i].v[7], scale, 3);
        } else {
            scale_bits = int4_scale_bits(m);
            const float s = bf16_bits_to_f32(scale_bits);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                code |= (uint32_t)(s > 0.0f ? int4_code(e[i].v[j], s) : 8) << (4 * j);
        }
        reinterpret_cast<uint32_t *>(g.codes)[(u[i].row * g.cols + u[i].col) / 8] = code;
        if (u[i].col % g.group == 0) {
            const int64_t at = u[i].row * g.scale_cols + u[i].col / g.group;
            if constexpr (kFormat == MOE_Q4_FP4)
                g.scales[at] = (unsigned char)scale_bits;
            else
                reinterpret_cast<uint16_t *>(g.scales)[at] = (uint16_t)scale_bits;
        }
    }
#endif
}

template <int kFormat, bool kBf16>
__global__ __launch_bounds__(kQ4Threads) void q4_dequantize(Q4Args g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const Q4Walk walk(g);
    uint32_t code[kQ4Per];
    float scale[kQ4Per];
    Q4Unit u[kQ4Per];
#pragma unroll
    for (int i = 0; i < kQ4Per; ++i) {
        u[i] = walk.at(i);
        code[i] = 0;
        scale[i] = 0.0f;
        if (u[i].row < g.rows && u[i].col < g.cols) {
            code[i] = reinterpret_cast<const uint32_t *>(g.codes)[(u[i].row * g.cols + u[i].col) / 8];
            const int64_t at = u[i].row * g.scale_cols + u[i].col / g.group;
            if constexpr (kFormat == MOE_Q4_FP4)
                scale[i] = fp4_scale(g.scales[at]);
            else
                scale[i] = bf16_bits_to_f32(reinterpret_cast<const uint16_t *>(g.scales)[at]);
        }
    }
#pragma unroll
    for (int i = 0; i < kQ4Per; ++i) {
        if (!(u[i].row < g.rows && u[i].col < g.cols))
            continue;
        float v[8];
        q4_values<kFormat>(code[i], scale[i], v);
        const int64_t at = u[i].row * g.cols + u[i].col;
        if constexpr (kBf16) {
            const u32x4 out = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
            __builtin_nontemporal_store(out, reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(g.w_out) + at));
        } else {
            f32x4 *const p = reinterpret_cast<f32x4 *>(static_cast<float *>(g.w_out) + at);
            const f32x4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
            __builtin_nontemporal_store(a, p);
            __builtin_nontemporal_store(b, p + 1);
        }
    }
#endif
}

static Q4Args q4_args(int64_t rows, int64_t cols, int group)
{
    Q4Args g = {};
    g.rows = rows;
    g.cols = (int)cols;
    g.group = cols < group ? (int)cols : group; // (64 columns under a scale for 128: as many lanes as there are columns)
    g.scale_cols = (int)q4_scale_cols(cols, group);
    g.units = g.scale_cols * (g.group / 8); // (at most 4/3 of the columns: a grid for 2^36 has fewer than 2^32 threads)
    return g;
}

int launch_quantize_q4(const void *w, int dtype, int64_t rows, int64_t cols, int format, int group, void *codes, void *scales,
                       hipStream_t st)
{
    Q4Args g = q4_args(rows, cols, group);
    g.w_in = w;
    g.codes = static_cast<unsigned char *>(codes);
    g.scales = static_cast<unsigned char *>(scales);
    const dim3 grid((unsigned)ceil_div(rows * g.units, kQ4Threads * kQ4Per)), block(kQ4Threads);
    auto kern = format == MOE_Q4_FP4 ? (dtype == MOE_BF16 ? q4_quantize<MOE_Q4_FP4, true> : q4_quantize<MOE_Q4_FP4, false>)
                                     : (dtype == MOE_BF16 ? q4_quantize<MOE_Q4_INT4, true> : q4_quantize<MOE_Q4_INT4, false>);
    hipLaunchKernelGGL(kern, grid, block, 0, st, g);
    return check_launch("moe_quantize_q4");
}

int launch_dequantize_q4(const void *codes, const void *scales, int format, int group, int64_t rows, int64_t cols, void *w,
                         int dtype, hipStream_t st)
{
    Q4Args g = q4_args(rows, cols, group);
    g.w_out = w;
    g.codes = static_cast<unsigned char *>(const_cast<void *>(codes));
    g.scales = static_cast<unsigned char *>(const_cast<void *>(scales));
    const dim3 grid((unsigned)ceil_div(rows * g.units, kQ4Threads * kQ4Per)), block(kQ4Threads);
    auto kern = format == MOE_Q4_FP4 ? (dtype == MOE_BF16 ? q4_dequantize<MOE_Q4_FP4, true> : q4_dequantize<MOE_Q4_FP4, false>)
                                     : (dtype == MOE_BF16 ? q4_dequantize<MOE_Q4_INT4, true> : q4_dequantize<MOE_Q4_INT4, false>);
    hipLaunchKernelGGL(kern, grid, block, 0, st, g);
    return check_launch("moe_dequantize_q4");
}

}  // namespace moe

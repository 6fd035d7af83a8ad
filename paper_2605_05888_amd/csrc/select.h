// Top-K selection and normalisation of one token's logits by one wavefront: moe_route's selection kernel and the decoding
// layer share it, so that both give the same bits.
#pragma once

#include <math.h>

#include <type_traits>

#include "common.h"

namespace moe {

// Value of the lane `kRor` places away inside a row of sixteen lanes.
template <int kRor, class T>
__device__ __forceinline__ T row_ror(T v)
{
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + kRor, 0xf, 0xf, true));
}
__device__ __forceinline__ float row_max16(float v)
{
    v = fmaxf(v, row_ror<8>(v));
    v = fmaxf(v, row_ror<4>(v));
    v = fmaxf(v, row_ror<2>(v));
    return fmaxf(v, row_ror<1>(v));
}
__device__ __forceinline__ float row_sum16(float v)
{
    v += row_ror<8>(v);
    v += row_ror<4>(v);
    v += row_ror<2>(v);
    return v + row_ror<1>(v);
}

__device__ __forceinline__ float score(float logit, float top, int score_mode)
{
    return score_mode == MOE_SCORE_SOFTMAX_TOPK ? expf(logit - top) : 1.0f / (1.0f + expf(-logit));
}

// lane 63's copy after folding all rows into it, for every lane
__device__ __forceinline__ float wave_max(float v)
{
    v = row_max16(v);
    auto move = [](float f, auto ctrl, auto rows) { // rows that do not take part keep their own value
        const int i = __builtin_bit_cast(int, f);
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
    };
    v = fmaxf(v, move(v, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{})); // row_bcast:15
    v = fmaxf(v, move(v, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{})); // row_bcast:31
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// Lane k < K: the k-th pick and its weight.
struct Pick {
    int expert;
    float weight;
};

// Selection.  One wavefront per token, lane l holds experts l, l+64, ... (kPer of them).  A round takes the
// largest value over the wavefront by data-parallel-primitive moves (no LDS), then the lowest index that has it
// (experts in ascending order are ballots of ascending i, lanes from the lowest).
// The K picks are distinct experts of [0, E) whatever the logits are: an overflowed token has infinities or NaN, a
// masked expert a bias of -infinity.  NaN counts as -infinity, so NaN can stand for "taken" and "not there": it never is
// the maximum as long as an expert is left (K <= E), and never equals it.  (With these in a bit mask beside the values:
// 1 token, 1024 experts, top-32 43 us instead of 33.)
// logit_of(e): expert e's logit, on the lane that asks.
template <int kPer, class LogitOf>
__device__ __forceinline__ Pick select_top(LogitOf logit_of, int E, int K, int score_mode)
{
    const int lane = threadIdx.x % kWave;
    float val[kPer]; // NaN: taken, or not there
    bool odd = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = i * kWave + lane;
        const float f = e < E ? logit_of(e) : 0.0f;
        odd |= f != f;
        val[i] = e < E ? (f == f ? f : -INFINITY) : NAN;
    }
    float my_logit = 0.0f, top = 0.0f; // lane k keeps the k-th pick
    int my_pick = 0;
    for (int k = 0; k < K; ++k) {
        float best = val[0];
#pragma unroll
        for (int i = 1; i < kPer; ++i)
            best = fmaxf(best, val[i]);
        best = wave_max(best);
        int pick = -1;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint64_t m = __ballot(val[i] == best);
            if (pick < 0 && m != 0) {
                const int at = __builtin_ctzll(m);
                pick = i * kWave + at;
                if (lane == at)
                    val[i] = NAN;
            }
        }
        if (k == 0)
            top = best;
        if (lane == k) {
            my_logit = best;
            my_pick = pick;
        }
    }
    if (__ballot(odd) != 0) { // the weights are those of the logits themselves
        my_logit = lane < K ? logit_of(my_pick) : 0.0f;
        top = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(my_logit), 0));
    }
    const float s = lane < K ? score(my_logit, top, score_mode) : 0.0f;
    // Sum in pairs of ranks that are 16, 8, 4, 2, 1 apart (K <= 32: the first two rows of sixteen lanes)
    const float pairs = K > 16 ? s + __shfl_xor(s, 16) : s;
    float sum = row_sum16(pairs);
    sum = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(sum), 0));
    return {my_pick, s / sum};
}

}  // namespace moe

// The decoding operators (few.hip, q4.hip), as api.hip sees them.
#pragma once

#include "../../include/moe_few.h"
#include "common.h"

namespace moe {

constexpr int64_t kFewMaxCols = (int64_t)1 << 21; // of H, F and the columns of 4-bit weights
constexpr int kNoFormat = -1; // weights in the activations' dtype

struct FewMatrix {
    const void *data;   // values, or codes
    const void *scales; // nullptr: values
};

struct FewArgs {
    const void *x;
    const float *W_r, *bias;
    FewMatrix gate, up, down;
    int32_t *topk_idx;
    float *topk_w;
    void *out;
    void *ws;
    void *a; // activation [N * K, F], in the workspace
    int N, H, E, K, F, score_mode;
    int group, scale_cols_h, scale_cols_f;
};

struct MatvecArgs {
    const void *x;
    FewMatrix w;
    void *y;
    const int32_t *seg_offsets;
    int64_t M, rows;
    int cols, group, scale_cols;
};

// Not part of the interface: what tests make of a wait of moe_layer_few.  polls: how often it looks before it takes over what
// is missing (0: at once; negative: as the library has it).  workgroups: how many are launched; fewer than one per compute unit
// (0: that) are what a call has while others hold the compute units.
extern "C" void moe_few_test_waits(int polls, int workgroups);

size_t few_workspace_bytes(int64_t N, int64_t H, int E, int K, int64_t F, int dtype);
int launch_layer_few(const FewArgs &args, int dtype, int format, hipStream_t st);
int launch_matvec_q4(const MatvecArgs &args, int E_local, int format, hipStream_t st);
int launch_quantize_q4(const void *w, int dtype, int64_t rows, int64_t cols, int format, int group, void *codes, void *scales,
                       hipStream_t st);
int launch_dequantize_q4(const void *codes, const void *scales, int format, int group, int64_t rows, int64_t cols, void *w,
                         int dtype, hipStream_t st);

}  // namespace moe

// few_ffn for fp32 weights and activations.
#include "few_ffn.h"

namespace moe {
template void launch_few_ffn<kFewF32>(const FewKernelArgs &g, hipStream_t st);
}  // namespace moe

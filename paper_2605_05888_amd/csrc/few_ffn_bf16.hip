// few_ffn for bf16 weights.
#include "few_ffn.h"

namespace moe {
template void launch_few_ffn<kFewBf16>(const FewKernelArgs &g, hipStream_t st);
}  // namespace moe

// few_ffn for FP4 weights.
#include "few_ffn.h"

namespace moe {
template void launch_few_ffn<kFewFp4>(const FewKernelArgs &g, hipStream_t st);
}  // namespace moe

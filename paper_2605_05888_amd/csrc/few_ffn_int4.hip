// few_ffn for INT4 weights.
#include "few_ffn.h"

namespace moe {
template void launch_few_ffn<kFewInt4>(const FewKernelArgs &g, hipStream_t st);
}  // namespace moe

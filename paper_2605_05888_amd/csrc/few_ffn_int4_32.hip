// few_ffn for INT4 weights, a scale for 32 columns.
#include "few_ffn.h"

namespace moe {
template void launch_few_ffn<kFewInt4By32>(const FewKernelArgs &g, hipStream_t st);
}  // namespace moe

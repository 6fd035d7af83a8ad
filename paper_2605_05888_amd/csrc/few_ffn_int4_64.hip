// few_ffn for INT4 weights, a scale for 64 columns.
#include "few_ffn.h"

namespace moe {
template void launch_few_ffn<kFewInt4By64>(const FewKernelArgs &g, hipStream_t st);
}  // namespace moe

// Attention on bf16 tensors, backward.
#include "attention_launch.h"

namespace lcn {
template hipError_t attention_backward<__bf16>(AttentionArgs, bool, int, hipStream_t);
}  // namespace lcn

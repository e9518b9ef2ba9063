// Attention on bf16 tensors, forward.
#include "attention_launch.h"

namespace lcn {
template hipError_t attention_forward<__bf16>(AttentionArgs, bool, int, hipStream_t);
template hipError_t attention_by_chunks<__bf16>(AttentionArgs, bool, int, hipStream_t);
}  // namespace lcn

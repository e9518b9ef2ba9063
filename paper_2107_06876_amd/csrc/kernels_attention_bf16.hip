// Attention on bf16 tensors.
#include "attention_launch.h"

namespace lcn {
template hipError_t attention_forward<__bf16>(AttentionArgs, bool, bool, hipStream_t);
template hipError_t attention_by_chunks<__bf16>(AttentionArgs, bool, bool, hipStream_t);
template hipError_t attention_backward<__bf16>(AttentionArgs, bool, bool, float *, const __bf16 *, hipStream_t);
}  // namespace lcn

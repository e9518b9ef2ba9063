// Attention on float tensors.
#include "attention_launch.h"

namespace lcn {
template hipError_t attention_forward<float>(AttentionArgs, bool, bool, hipStream_t);
template hipError_t attention_by_chunks<float>(AttentionArgs, bool, bool, hipStream_t);
template hipError_t attention_backward<float>(AttentionArgs, bool, bool, float *, const float *, hipStream_t);
}  // namespace lcn

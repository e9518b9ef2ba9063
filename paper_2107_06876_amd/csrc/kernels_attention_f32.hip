// Attention on float tensors, forward.
#include "attention_launch.h"

namespace lcn {
template hipError_t attention_forward<float>(AttentionArgs, bool, int, hipStream_t);
template hipError_t attention_by_chunks<float>(AttentionArgs, bool, int, hipStream_t);
}  // namespace lcn

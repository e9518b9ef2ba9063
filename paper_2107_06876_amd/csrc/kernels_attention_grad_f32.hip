// Attention on float tensors, backward.
#include "attention_launch.h"

namespace lcn {
template hipError_t attention_backward<float>(AttentionArgs, bool, int, hipStream_t);
}  // namespace lcn

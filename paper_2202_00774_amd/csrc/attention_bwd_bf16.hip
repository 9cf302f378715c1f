// The kernels of attention's gradients on bf16 tensors.
#include "attention_bwd_launch.h"

namespace sdgp {
template int attention_bwd_launch<SDGP_BF16>(Attention a, const AttentionGrid& g, hipStream_t stream);
}  // namespace sdgp

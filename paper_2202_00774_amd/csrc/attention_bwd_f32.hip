// The kernels of attention's gradients on fp32 tensors.
#include "attention_bwd_launch.h"

namespace sdgp {
template int attention_bwd_launch<SDGP_F32>(Attention a, const AttentionGrid& g, hipStream_t stream);
}  // namespace sdgp

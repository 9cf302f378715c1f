// The forward attention kernels on fp32 tensors.
#include "attention_fwd_launch.h"

namespace sdgp {
template int attention_fwd_launch<SDGP_F32>(const Attention& a, int64_t tiles, bool few, hipStream_t stream);
}  // namespace sdgp

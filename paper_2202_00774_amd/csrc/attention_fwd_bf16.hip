// The forward attention kernels on bf16 tensors.
#include "attention_fwd_launch.h"

namespace sdgp {
template int attention_fwd_launch<SDGP_BF16>(const Attention& a, int64_t tiles, bool few, hipStream_t stream);
}  // namespace sdgp

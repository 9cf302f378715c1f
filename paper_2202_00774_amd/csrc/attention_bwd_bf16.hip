// The kernels of attention's gradients on bf16 tensors.
#include "attention_bwd_launch.h"

namespace sdgp {
template int attention_bwd_launch<SDGP_BF16>(const Attention& a, int64_t row_tiles, int64_t key_tiles, hipStream_t stream);
}  // namespace sdgp

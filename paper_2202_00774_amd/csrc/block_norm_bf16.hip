// Block norms of bf16 rows (block_norm_rows.h).
#include "block_norm_rows.h"

namespace sdgp {
template int norm_rows_launch<SDGP_BF16>(const Norm& n, RowShape shape, hipStream_t stream);
template int norm_grad_launch<SDGP_BF16>(const NormGrad& n, RowShape shape, hipStream_t stream);
}  // namespace sdgp

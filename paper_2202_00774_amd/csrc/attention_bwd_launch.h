// Launches of the kernels of attention's gradients.
#pragma once

#include "attention_bwd.h"

namespace sdgp {

template <int DT>
int attention_bwd_launch(const Attention& a, int64_t row_tiles, int64_t key_tiles, hipStream_t stream) {
    const dim3 block(256);
    int rc = SDGP_OK;
    const auto launch = [&](auto width, auto fast) {
        constexpr int DC = decltype(width)::value;
        constexpr bool FAST = decltype(fast)::value;
        if (row_tiles > 0) hipLaunchKernelGGL((attention_dq_kernel<DT, DC, FAST>), dim3((unsigned)(row_tiles * a.Hk)), block, 0, stream, a);
        rc = launch_status();
        if (rc != SDGP_OK || key_tiles == 0) return;
        hipLaunchKernelGGL((attention_dkv_kernel<DT, DC, FAST>), dim3((unsigned)(key_tiles * a.Hk)), block, 0, stream, a);
        rc = launch_status();
    };
    if (!a.fast) launch(std::integral_constant<int, 128>{}, std::false_type{});
    else if (a.D <= 64) launch(std::integral_constant<int, 64>{}, std::true_type{});
    else if (a.D <= 96) launch(std::integral_constant<int, 96>{}, std::true_type{});
    else launch(std::integral_constant<int, 128>{}, std::true_type{});
    return rc;
}

}  // namespace sdgp

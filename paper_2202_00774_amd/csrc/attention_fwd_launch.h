// Launches of the forward attention kernels.
#pragma once

#include "attention_fwd.h"

namespace sdgp {

template <int DT>
int attention_fwd_launch(const Attention& a, int64_t tiles, bool few, hipStream_t stream) {
    const dim3 grid((unsigned)(tiles * a.Hk * a.parts)), block(256);
    const auto launch = [&](auto width, auto fast) {
        constexpr int DC = decltype(width)::value;
        constexpr bool FAST = decltype(fast)::value;
        if (few) hipLaunchKernelGGL((attention_fwd_kernel<DT, DC, true, FAST>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((attention_fwd_kernel<DT, DC, false, FAST>), grid, block, 0, stream, a);
    };
    if (!a.fast) launch(std::integral_constant<int, 128>{}, std::false_type{});
    else if (a.D <= 64) launch(std::integral_constant<int, 64>{}, std::true_type{});
    else if (a.D <= 96) launch(std::integral_constant<int, 96>{}, std::true_type{});
    else launch(std::integral_constant<int, 128>{}, std::true_type{});
    const int rc = launch_status();
    if (rc != SDGP_OK || a.parts == 1) return rc;
    hipLaunchKernelGGL((attention_join<DT>), dim3((unsigned)(((int64_t)a.Tq * a.H + 3) / 4)), block, 0, stream, a);
    return launch_status();
}

}  // namespace sdgp

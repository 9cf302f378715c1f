// Launches of the kernels of attention's gradients.
#pragma once

#include "attention_bwd.h"

namespace sdgp {

template <int DT>
int attention_bwd_launch(Attention a, const AttentionGrid& g, hipStream_t stream) {
    const dim3 block(256);
    int rc = SDGP_OK;
    const int parts = a.parts;
    const auto launch = [&](auto width, auto fast) {
        constexpr int DC = decltype(width)::value;
        constexpr bool FAST = decltype(fast)::value;
        if (g.row_tiles > 0) {
            const dim3 grid((unsigned)(g.row_tiles * a.Hk));
            if (g.own_rows == 4) hipLaunchKernelGGL((attention_dq_kernel<DT, DC, FAST, 4>), grid, block, 0, stream, a);
            else hipLaunchKernelGGL((attention_dq_kernel<DT, DC, FAST, 2>), grid, block, 0, stream, a);
            rc = launch_status();
        }
        if (rc != SDGP_OK || g.key_tiles == 0) return;
        hipLaunchKernelGGL((attention_dkv_kernel<DT, DC, FAST, attention_own_keys(DT)>), dim3((unsigned)(g.key_tiles * a.Hk * parts)), block, 0, stream, a);
        rc = launch_status();
    };
    if (!a.fast) launch(std::integral_constant<int, 128>{}, std::false_type{});
    else if (a.D <= 64) launch(std::integral_constant<int, 64>{}, std::true_type{});
    else if (a.D <= 96) launch(std::integral_constant<int, 96>{}, std::true_type{});
    else launch(std::integral_constant<int, 128>{}, std::true_type{});
    if (rc != SDGP_OK || parts == 1 || g.key_tiles == 0) return rc;
    const int64_t values = 2 * (int64_t)a.Tk * a.Hk * a.D, blocks = (values + 1023) / 1024 + 1;
    hipLaunchKernelGGL((attention_dkv_join<DT>), dim3((unsigned)(blocks < 16384 ? blocks : 16384)), block, 0, stream, a);
    return launch_status();
}

}  // namespace sdgp

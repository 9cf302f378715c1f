"""Attention of values as large as the header allows: its sums run over exp(s - m) v, where m may stay 8 ln 2 behind a row's maximum."""
import math

import pytest
import torch

import paper_2202_00774_amd as sdgp
from attention_reference import attention, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("queries, keys", [(1, 512), (40, 512), (1, 65536), (200, 4096)])
@pytest.mark.parametrize("signs", [True, False])
def test_values_up_to_the_bound(queries, keys, signs, dtype):
    """Scores of 0 in front and 7.9 ln 2 behind: m stays at 0, so nearly all terms are 2^7.9 v.  |v| keys = 2^119."""
    H, D = 2, 64
    q, k = torch.zeros(queries, H, D, dtype=dtype, device="cuda"), torch.zeros(keys, H, D, dtype=dtype, device="cuda")
    q[..., 0], k[64:, :, 0] = 1.0, 7.9
    v = torch.full((keys, H, D), 2.0 ** 119 / keys, dtype=dtype, device="cuda")
    if signs:
        v[::2] *= -1
        v[keys // 2:] *= 0.25
    ref = attention(q, k, v, [(0, queries, 0, keys)], False, math.log(2.0))
    o, lse = sdgp.sdgp_attention(q[None], k[None], v[None], causal=False, scale=math.log(2.0))
    check(o[0], ref, "o")
    check(lse[0], ref, "lse")

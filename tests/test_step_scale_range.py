"""The scale's range, at the C boundary without a GPU: scale * log2(e) has to have an fp32 value, or every number of every row
would be NaN (0 times infinity at the row's largest logit)."""
import ctypes

import pytest

from paper_2202_00774_amd import binding

P, VALUE = ctypes.c_void_p(16), -8       # never dereferenced: every call is refused


@pytest.mark.parametrize("scale", [1.8e38, 2.4e38, 3.4028234e38])
def test_scales_above_2_to_127_are_refused(scale):
    lib = binding.load()
    assert lib.sdgp_token_logprobs(P, 16, P, 64, P, P, P, P, P, 2, 16, 1, 4, scale, P, 1 << 30, None) == VALUE
    assert lib.sdgp_token_logprobs_bwd(P, 16, P, 64, P, P, P, P, P, 16, 2, 16, 1, scale, None) == VALUE

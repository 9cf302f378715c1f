"""The losses over sequences at their edges: no sequences, and terms that add up beyond 32 bits."""
import math

import pytest
import torch

import paper_2202_00774_amd as sdgp

pytestmark = pytest.mark.gpu
F = 2.0 ** -24


# One launch takes up to 4096 tokens of the policy loss and 16384 of the preference loss; above, sequences have a launch of their own.
@pytest.mark.parametrize("T", [0, 8, 4096, 4097, 5000, 16385, 20000])
@pytest.mark.parametrize("first", [0, 7])
def test_no_sequences(T, first):
    """Offsets of one entry: no token counts, so the losses and gradients are 0 whatever stands there."""
    logp, old, ref = (torch.full((T,), math.nan, device="cuda") for _ in range(3))
    offsets, g = torch.tensor([first], dtype=torch.int32, device="cuda"), torch.ones((), device="cuda")
    for average in ("tokens", "sequences"):
        for adv in (torch.full((T,), math.nan, device="cuda"), torch.empty(0, device="cuda")):
            how = {"kl": 0.5, "average": average}
            *out, weights = sdgp.sdgp_policy_loss(logp, old, adv, ref, None, offsets, **how)
            assert [x.item() for x in out] == [0.0, 0.0, 0.0] and weights.shape == (0,)
            assert not sdgp.sdgp_policy_loss_bwd(g, weights, logp, old, adv, ref, None, offsets, **how).any()
    loss, margins, weights = sdgp.sdgp_preference_loss(logp, ref, None, offsets)
    assert loss.item() == 0.0 and margins.shape == weights.shape == (0,)
    assert not sdgp.sdgp_preference_loss_bwd(g, weights, logp, None, offsets).any()


@pytest.mark.parametrize("T", [4, 255, 5000])
def test_terms_that_pass_32_bits_together(T):
    """Terms of e^88 = 1.65e38 each: any three of them pass 3.4e38, their mean does not."""
    logp = torch.full((T,), -100.0, device="cuda")
    zero, twelve = torch.zeros(T, device="cuda"), torch.full((T,), -12.0, device="cuda")
    want = math.exp(88.0)
    # e^x is off by 2 steps (4 F) of itself at most, storing by F; nothing else here rounds by more than 2^-50
    loss, kl, _, _ = sdgp.sdgp_policy_loss(logp, logp, zero, twelve, kl=1.0)
    assert abs(kl.item() - want) <= 5 * F * want and abs(loss.item() - want) <= 5 * F * want
    loss, _, clipped, _ = sdgp.sdgp_policy_loss(twelve, logp, zero - 1.0)
    assert abs(loss.item() - want) <= 5 * F * want and clipped.item() == 0.0


def test_terms_of_both_signs_lose_nothing():
    """A lane's four terms: 2^24, 1, -2^24, 1 have a mean of 1/2, whatever 32 bits would leave of it."""
    z = torch.zeros(4, device="cuda")
    adv = torch.tensor([-(2.0 ** 24), -1.0, 2.0 ** 24, -1.0], device="cuda")
    loss, _, _, _ = sdgp.sdgp_policy_loss(z, z, adv)
    assert loss.item() == 0.5

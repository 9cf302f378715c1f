"""Arguments of the token log probabilities that a call does not need, and values at the ends of their ranges."""
import pytest
import torch

import paper_2202_00774_amd as sdgp
from paper_2202_00774_amd.autograd import sdgp_token_logprobs

pytestmark = pytest.mark.gpu


def test_entropy_alone_with_32_bit_tokens_that_start_anywhere():
    """The gradient through the entropy reads no tokens, so it is the same whatever they are and wherever they start."""
    x = torch.randn(5, 300, device="cuda")
    room = torch.randint(0, 300, (8,), device="cuda", dtype=torch.int32)
    want = None
    for tokens in (None, room[:5], room[1:6], room[2:7], room[3:8].long()):
        leaf = x.clone().requires_grad_()
        sdgp_token_logprobs(leaf, tokens)[1].sum().backward()
        want = leaf.grad if want is None else want
        assert torch.equal(leaf.grad, want)
    _, entropy, _, _, stats = sdgp.sdgp_token_logprobs(x, room[1:6])
    assert torch.equal(sdgp.sdgp_token_logprobs_bwd(x, room[1:6], stats, entropy, None, torch.ones(5, device="cuda")), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [9, 300, 9001])
def test_a_token_outside_the_vocabulary_of_a_row_that_leaves_nothing(dtype, V):
    """NaN, forward and in the gradient, as in any other row: what is not a token is not an empty row's business."""
    x = torch.full((4, V), -float("inf"), device="cuda", dtype=dtype)
    x[3] = 1.0
    tokens = torch.tensor([V, 0, -1, V + 5], device="cuda")
    logp, entropy, _, _, stats = sdgp.sdgp_token_logprobs(x, tokens)
    assert torch.equal(torch.isnan(logp), torch.tensor([True, False, False, True], device="cuda")) and logp[1] == -float("inf") and logp[2] == 0
    g = torch.ones(4, device="cuda")
    for h in (None, g):
        d = sdgp.sdgp_token_logprobs_bwd(x, tokens, stats, entropy, g, h)
        assert torch.isnan(d[0]).all() and (d[1:3] == 0).all() and torch.isnan(d[3]).all()
    assert (sdgp.sdgp_token_logprobs_bwd(x, tokens, stats, entropy, None, g)[:3] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_largest_and_smallest_scales(dtype):
    """2^127: all of the probability is the largest logit's, shared by equal ones.  2^-149: all tokens are alike."""
    x = torch.tensor([[1.0, 3.0, -2.0, 3.0], [0.5, -0.5, 0.25, -1.0], [-float("inf"), 7.0, 1.0, 2.0]], device="cuda").to(dtype)
    tokens = torch.tensor([1, 0, 1], device="cuda")
    for wide in (1, 1500):                                       # one chunk, several
        at = torch.cat([x] + [torch.full((3, 1), torch.finfo(dtype).min, device="cuda", dtype=dtype).expand(3, 4)] * (wide - 1), 1)
        logp, entropy, top_logp, top_ids, stats = sdgp.sdgp_token_logprobs(at, tokens, top=2, scale=2.0 ** 127)
        ln2 = torch.tensor(2.0).log()
        assert (logp.cpu() - torch.tensor([-ln2, 0, 0])).abs().max() <= 1e-6 and (entropy.cpu() - torch.tensor([ln2, 0, 0])).abs().max() <= 1e-6
        assert top_ids[0].tolist() == [1, 3] and top_ids[1:, 0].tolist() == [0, 1]
        d = sdgp.sdgp_token_logprobs_bwd(at, tokens, stats, entropy, torch.full((3,), 2.0 ** -126, device="cuda"), None, scale=2.0 ** 127)
        want = torch.zeros_like(at)
        want[0, 1], want[0, 3] = 1.0, -1.0
        assert (d.float() - want.float()).abs().max() <= 2.0 ** -7
    logp, entropy, _, _, _ = sdgp.sdgp_token_logprobs(x[:2], tokens[:2], scale=2.0 ** -149)
    assert (logp + 2 * ln2).abs().max() <= 1e-6 and (entropy - 2 * ln2).abs().max() <= 1e-6

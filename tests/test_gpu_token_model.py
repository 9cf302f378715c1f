"""The loss, norm and optimizer operators together, and their autograd functions."""
import importlib.util
import os

import pytest
import torch

import paper_2202_00774_amd as sdgp
from paper_2202_00774_amd.autograd import sdgp_block_norm, sdgp_linear, sdgp_token_logprobs

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("token_model", os.path.join(ROOT, "examples", "token_model.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def composed_norm(x, u, gate, w_post, w_pre, residual_scale, eps=1e-6):
    norm = lambda v: v * torch.rsqrt((v * v).mean(-1, keepdim=True) + eps)  # noqa: E731
    y = x if u is None else residual_scale * x + gate * (norm(u) * w_post)
    return y, norm(y) * w_pre


def test_block_norm_gradients_agree_with_torch():
    """fp32 against the same formula in float64 by torch's own autograd: both are the gradient, so they agree to the rounding
    of sums over 96 values and 30 rows: 1e-5 of the largest."""
    torch.manual_seed(0)
    shapes = {"x": (5, 6, 96), "u": (5, 6, 96), "gate": (5, 1, 96), "w_post": (96,), "w_pre": (96,)}
    own = {k: torch.randn(s, device="cuda").requires_grad_() for k, s in shapes.items()}
    ref = {k: v.detach().double().requires_grad_() for k, v in own.items()}
    y, h = sdgp_block_norm(*own.values(), residual_scale=0.8)
    ry, rh = composed_norm(*ref.values(), 0.8)
    a, b = torch.randn_like(y), torch.randn_like(y)
    ((y * a).sum() + (h * b.transpose(0, 1).contiguous().transpose(0, 1)).sum()).backward()
    ((ry * a.double()).sum() + (rh * b.double()).sum()).backward()
    assert torch.allclose(y.double(), ry, atol=1e-5) and torch.allclose(h.double(), rh, atol=1e-5)
    for k in shapes:
        g, r = own[k].grad.double(), ref[k].grad
        assert g.shape == r.shape and (g - r).abs().max() <= 1e-5 * r.abs().max(), k


def test_block_norm_without_a_block_and_one_output_unused():
    torch.manual_seed(1)
    x = torch.randn(7, 40, device="cuda").requires_grad_()
    w = torch.randn(40, device="cuda").requires_grad_()
    y, h = sdgp_block_norm(x, w_pre=w)
    assert y is x
    (y.sum() + (h * h).sum()).backward()
    xr, wr = x.detach().double().requires_grad_(), w.detach().double().requires_grad_()
    yr, hr = composed_norm(xr, None, None, None, wr, 1.0)
    (yr.sum() + (hr * hr).sum()).backward()
    assert (x.grad - xr.grad).abs().max() <= 1e-5 * xr.grad.abs().max() and (w.grad - wr.grad).abs().max() <= 1e-5 * wr.grad.abs().max()
    # only y goes on, only h goes on, no norm follows
    u = torch.randn(7, 40, device="cuda").requires_grad_()
    for pick in (0, 1):
        x.grad = u.grad = None
        sdgp_block_norm(x, u)[pick].sum().backward()
        xr, ur = x.detach().double().requires_grad_(), u.detach().double().requires_grad_()
        composed_norm(xr, ur, 1.0, 1.0, 1.0, 1.0)[pick].sum().backward()
        for g, r in ((x.grad, xr.grad), (u.grad, ur.grad)):
            assert (g - r).abs().max() <= 1e-5 * max(1.0, r.abs().max().item())
    y, h = sdgp_block_norm(x, u, pre=False)
    assert h is None
    y.sum().backward()


def test_token_logprobs_gradients_agree_with_torch():
    torch.manual_seed(2)
    x = torch.randn(3, 4, 301, device="cuda").requires_grad_()
    tokens = torch.randint(0, 301, (3, 4), device="cuda")
    tokens[1, 2] = -100
    logp, entropy, top_logp, top_ids = sdgp_token_logprobs(x, tokens, top=3, scale=1.25)
    assert not top_logp.requires_grad and not top_ids.requires_grad and logp.requires_grad
    (-logp.mean() - 0.1 * entropy.mean()).backward()
    r = x.detach().double().requires_grad_()
    q = torch.log_softmax(1.25 * r, -1)
    picked = torch.where(tokens >= 0, q.gather(-1, tokens.clamp(min=0)[..., None])[..., 0], 0.0)
    (-picked.mean() + 0.1 * (q.exp() * q).sum(-1).mean()).backward()
    assert (x.grad - r.grad).abs().max() <= 1e-5 * r.grad.abs().max()
    # one of the two outputs, and no tokens
    x.grad = None
    sdgp_token_logprobs(x, None)[1].sum().backward()
    r.grad = None
    q = torch.log_softmax(r, -1)
    (-(q.exp() * q).sum(-1)).sum().backward()
    assert (x.grad - r.grad).abs().max() <= 1e-5 * r.grad.abs().max()


def test_the_gradient_is_what_the_last_layer_prunes():
    """dL/dlogits goes into the pruned backward pass as any dL/dO: the input gradient is the library's own product of it."""
    torch.manual_seed(3)
    h = torch.randn(33, 64, device="cuda", dtype=torch.bfloat16).requires_grad_()
    w = torch.randn(100, 64, device="cuda", dtype=torch.bfloat16)
    tokens = torch.randint(0, 100, (33,), device="cuda")
    logits = sdgp_linear(h, w, 2, 4, sdgp.GREEDY)
    sdgp_token_logprobs(logits, tokens)[0].sum().backward()
    _, _, _, _, stats = sdgp.sdgp_token_logprobs(logits.detach(), tokens)
    dO = sdgp.sdgp_token_logprobs_bwd(logits.detach(), tokens, stats, None, torch.ones(33, device="cuda"))
    assert torch.equal(h.grad, sdgp.sdgp_linear_bwd_data(dO, w, 2, 4, sdgp.GREEDY))


@pytest.mark.parametrize("state_bits", [8, 32])
def test_the_model_learns_the_chain(state_bits):
    """From ln 500 = 6.2 nats to near the chain's own entropy of ln 4 = 1.39; then the four successors are its first four
    alternatives.  (A model that knew only which tokens are frequent would stay at 6.2.)"""
    m = example()
    model = m.TokenModel()
    losses = m.train(model, 200, state_bits)
    assert losses[0] > 5.5 and sum(losses[-10:]) / 10 < 1.8
    right = 0
    for token, ids, p in m.ask(model, 3, 8):
        assert abs(sum(p)) <= 1.0 + 1e-4 and p == sorted(p, reverse=True)
        right += len(set(ids[:4]) & {(7 * token + 1 + i) % m.VOCAB for i in range(4)})
    assert right >= 28
    for k, v in model.weights.items():
        assert torch.equal(v.detach(), model.masters[k].to(torch.bfloat16)), k


def test_a_captured_graph_replays_the_operators():
    """Loss, gradient and norms recorded once; every replay gives what the eager calls give on the inputs of the moment."""
    torch.manual_seed(5)
    x = torch.randn(6, 70001, device="cuda", dtype=torch.bfloat16)               # few long rows: two kernels and a workspace
    tokens = torch.randint(0, 70001, (6,), device="cuda")
    g = torch.randn(6, device="cuda")
    a, b = torch.randn(2, 300, 264, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(264, device="cuda")

    def work():
        logp, entropy, top_logp, top_ids, stats = sdgp.sdgp_token_logprobs(x, tokens, top=5)
        d = sdgp.sdgp_token_logprobs_bwd(x, tokens, stats, entropy, g, g)
        y, h, s = sdgp.sdgp_block_norm(a, b, None, w, w)
        return (logp, entropy, top_logp, top_ids, d, y, h, *(t for t in sdgp.sdgp_block_norm_bwd(a, b, y, s, b, None, w, w) if t is not None))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for i in range(4):
        x.copy_(torch.randn(x.shape, device="cuda"))
        a.copy_(torch.randn(a.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(held, work()):
            assert torch.equal(p, q), i

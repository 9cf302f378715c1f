"""Attention, positions and the losses as they are used together: gradients of a small model through all of them against 64
bits, differences of each operator's loss, captured graphs, other streams."""
import math

import pytest
import torch
import torch.nn.functional as F

import paper_2202_00774_amd as sdgp
from attention_reference import check, spans_of
from attention_reference import attention as attention_reference
from paper_2202_00774_amd import autograd as ag
from paper_2202_00774_amd.optim import AdamW

pytestmark = pytest.mark.gpu
LENS, VOCAB, WIDTH, H, HK, D = [17, 1, 40, 33], 50, 32, 4, 2, 8


def randn(seed, *shape):
    return torch.randn(*shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))


def batch():
    ends = [0]
    for n in LENS:
        ends.append(ends[-1] + n)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    T = ends[-1]
    tokens = torch.randint(0, VOCAB, (T,), device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    positions = torch.cat([torch.arange(n) for n in LENS]).cuda()
    return offsets, tokens, positions, T


def weights(dtype):
    shapes = {"embed": (VOCAB, WIDTH), "qkv": ((H + 2 * HK) * D, WIDTH), "out": (WIDTH, H * D), "head": (VOCAB, WIDTH)}
    return {k: (randn(i, *s) * s[-1] ** -0.5).to(dtype).requires_grad_() for i, (k, s) in enumerate(shapes.items())}


def own_logp(w, tokens, positions, offsets, freqs):
    x = F.embedding(tokens, w["embed"])
    y, h = ag.sdgp_block_norm(x)
    q, k, v = F.linear(h, w["qkv"]).view(-1, H + 2 * HK, D).split((H, HK, HK), 1)
    q, k = ag.sdgp_rotary(q, k, positions, freqs)
    o = ag.sdgp_attention(q, k, v, offsets)
    y, h = ag.sdgp_block_norm(y, F.linear(o.reshape(-1, H * D), w["out"]))
    return ag.sdgp_token_logprobs(F.linear(h, w["head"]), tokens.roll(-1))[0]


def plain_logp(w, tokens, positions, offsets, freqs):
    rms = lambda x: x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    x = w["embed"][tokens]
    q, k, v = (rms(x) @ w["qkv"].T).view(-1, H + 2 * HK, D).split((H, HK, HK), 1)
    angle = positions[:, None, None].double() * freqs.double()
    turn = lambda z: torch.cat([z[..., :D // 2] * angle.cos() - z[..., D // 2:] * angle.sin(),  # noqa: E731
                                z[..., :D // 2] * angle.sin() + z[..., D // 2:] * angle.cos()], -1)
    q, k = turn(q), turn(k)
    rows = []
    for a, b in zip(offsets.tolist(), offsets.tolist()[1:]):
        hidden = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1)
        heads = [torch.softmax((q[a:b, h] @ k[a:b, h // (H // HK)].T * D ** -0.5).masked_fill(hidden, -math.inf), 1) @ v[a:b, h // (H // HK)]
                 for h in range(H)]
        rows.append(torch.stack(heads, 1))
    y = x + rms(torch.cat(rows).reshape(-1, H * D) @ w["out"].T)
    return torch.log_softmax(rms(y) @ w["head"].T, 1).gather(1, tokens.roll(-1)[:, None])[:, 0]


def losses(logp, offsets, plain):
    """A policy loss and a preference loss of the same log probabilities."""
    T = logp.numel()
    old = logp.detach() + 0.1 * randn(11, T).to(logp.dtype)
    ref, adv = logp.detach() + 0.2 * randn(12, T).to(logp.dtype), randn(13, len(LENS))
    if not plain:
        loss, _, _ = ag.sdgp_policy_loss(logp, old, adv, ref, None, offsets, clip=(0.05, 0.05), kl=0.3, average="sequences")
        return loss + ag.sdgp_preference_loss(logp, ref, None, offsets, beta=0.5)[0]
    ends = offsets.tolist()
    means, scores = [], []
    for i, (a, b) in enumerate(zip(ends, ends[1:])):
        r, x = torch.exp(logp[a:b] - old[a:b]), ref[a:b] - logp[a:b]
        means.append((0.3 * (torch.expm1(x) - x) - torch.minimum(r * adv[i], r.clamp(0.95, 1.05) * adv[i])).mean())
        scores.append(-0.5 * x.sum())
    z = torch.stack(scores).view(-1, 2)
    return torch.stack(means).mean() - F.logsigmoid(z[:, 0] - z[:, 1]).mean()


def test_gradients_of_a_model_in_fp32():
    """All roundings are 2^-24; a chain of a few hundred operations on values of about 1 keeps gradients to 1e-4 of their size
    (2^-24 times some hundred terms a sum times the chain's depth of about ten), the largest weight's gradient as the measure."""
    offsets, tokens, positions, T = batch()
    freqs = 50.0 ** (-torch.arange(D // 2, device="cuda") / (D // 2))
    w = weights(torch.float32)
    loss = losses(own_logp(w, tokens, positions, offsets, freqs), offsets, False)
    got = torch.autograd.grad(loss, list(w.values()))
    w64 = {k: v.detach().double().requires_grad_() for k, v in w.items()}
    loss64 = losses(plain_logp(w64, tokens, positions, offsets, freqs), offsets, True)
    want = torch.autograd.grad(loss64, list(w64.values()))
    assert abs(loss.item() - loss64.item()) <= 1e-4 * max(1.0, abs(loss64.item()))
    for a, b in zip(got, want):
        assert float((a - b).norm()) <= 1e-4 * float(b.norm())


def test_a_step_in_bf16():
    """Loss, gradients and an optimizer step on bf16 weights; the gradients of attention's part against 64 bits at the same inputs."""
    offsets, tokens, positions, T = batch()
    freqs = 50.0 ** (-torch.arange(D // 2, device="cuda") / (D // 2))
    w = weights(torch.bfloat16)
    masters = [p.detach().float() for p in w.values()]
    optimizer = AdamW(masters, copies=[p.detach() for p in w.values()], lr=1e-2)
    for _ in range(2):
        loss = losses(own_logp(w, tokens, positions, offsets, freqs), offsets, False)
        grads = torch.autograd.grad(loss, list(w.values()))
        assert all(bool(g.isfinite().all()) for g in grads)
        optimizer.step([g.contiguous() for g in grads])
    q, k, v = (randn(i, T, h, D).bfloat16().requires_grad_() for i, h in enumerate((H, HK, HK)))
    do = randn(9, T, H, D).bfloat16()
    o = ag.sdgp_attention(q, k, v, offsets)
    ref = attention_reference(q.detach(), k.detach(), v.detach(), spans_of(LENS, LENS), True, D ** -0.5, do)
    check(o.detach(), ref, "o")
    for name, t in zip(("dq", "dk", "dv"), torch.autograd.grad(o, (q, k, v), do)):
        check(t, ref, name)


def difference(f, x, direction, h):
    return (f(x + h * direction).item() - f(x - h * direction).item()) / (2 * h)


def test_gradients_against_differences():
    """Central differences of the fp32 operators along a direction: the third derivative's h^2 (about 1e-4 at h = 1e-2) and the
    roundings of two values of size F over 2 h, some 2^-20 F / h."""
    offsets, _, positions, T = batch()
    q, k, v, probe = (randn(i, T, h, D) for i, h in enumerate((H, HK, HK, H)))
    freqs = 50.0 ** (-torch.arange(D // 2, device="cuda") / (D // 2))
    for i in range(3):
        def f(x):
            given = [q, k, v]
            given[i] = x
            a, b = ag.sdgp_rotary(given[0], given[1], positions, freqs)
            return (ag.sdgp_attention(a, b, given[2], offsets) * probe).sum() / T

        x = (q, k, v)[i].clone().requires_grad_()
        g, = torch.autograd.grad(f(x), x)
        direction = randn(20 + i, *x.shape)
        direction /= direction.norm()
        want = difference(f, x.detach(), direction, 1e-1)
        assert abs(float((g * direction).sum()) - want) <= 1e-2 * float(g.norm()) * 0.1 + 2.0 ** -20 * 10


def test_captured_and_replayed():
    """Every call in one graph, replayed with other inputs and with eager work in between."""
    offsets, tokens, positions, T = batch()
    freqs = 50.0 ** (-torch.arange(D // 2, device="cuda") / (D // 2))
    q, k, v, do = (torch.zeros(T, h, D, device="cuda", dtype=torch.bfloat16) for h in (H, HK, HK, H))
    cache_k, cache_v, one = (torch.zeros(2, n, h, D, device="cuda", dtype=torch.bfloat16) for n, h in ((600, HK), (600, HK), (1, H)))
    lengths = torch.zeros(2, dtype=torch.int32, device="cuda")
    logp, old, ref = (torch.zeros(T, device="cuda") for _ in range(3))
    adv, g = torch.zeros(len(LENS), device="cuda"), torch.ones((), device="cuda")
    many = torch.zeros(20000, device="cuda")

    def all_calls():
        q2, k2 = sdgp.sdgp_rotary(q, k, positions, freqs)
        o, lse = sdgp.sdgp_attention(q2, k2, v, offsets)
        grads = sdgp.sdgp_attention_bwd(do, q2, k2, v, o, lse, offsets)
        decoded = sdgp.sdgp_attention(one, cache_k, cache_v, lengths=lengths)
        p = sdgp.sdgp_policy_loss(logp, old, adv, ref, None, offsets, kl=0.1)
        dp = sdgp.sdgp_policy_loss_bwd(g, p[-1], logp, old, adv, ref, None, offsets, kl=0.1)
        r = sdgp.sdgp_preference_loss(logp, ref, None, offsets)
        dr = sdgp.sdgp_preference_loss_bwd(g, r[-1], logp, None, offsets)
        long = sdgp.sdgp_policy_loss(many, many.roll(1), many[:1])
        return [q2, k2, o, lse, *grads, *decoded, *p, dp, *r, dr, *long]

    def fill(seed):
        for i, t in enumerate((q, k, v, do, cache_k, cache_v, one, logp, old, ref, adv, many)):
            t.copy_(randn(100 * seed + i, *t.shape))
        lengths.copy_(torch.tensor([37 * seed, 600 - seed], dtype=torch.int32))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = all_calls()
    for seed in (1, 2, 3):
        fill(seed)
        graph.replay()
        eager = all_calls()
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b) or torch.equal(a.isnan(), b.isnan()) and torch.equal(a[~a.isnan()], b[~b.isnan()])


def test_gradients_captured_and_replayed():
    """The model's forward pass, losses and their gradients in one graph; no eager graph of its weights lives meanwhile."""
    offsets, tokens, positions, T = batch()
    w = weights(torch.bfloat16)
    freqs = 50.0 ** (-torch.arange(D // 2, device="cuda") / (D // 2))
    old, ref, adv = (torch.zeros(n, device="cuda") for n in (T, T, len(LENS)))

    def step():
        logp = own_logp(w, tokens, positions, offsets, freqs)
        loss = ag.sdgp_policy_loss(logp, old, adv, ref, None, offsets, kl=0.1)[0] + ag.sdgp_preference_loss(logp, ref, None, offsets)[0]
        return [loss.detach(), *torch.autograd.grad(loss, list(w.values()))]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for seed in (1, 2, 3):
        for i, t in enumerate((old, ref, adv)):
            t.copy_(randn(10 * seed + i, *t.shape))
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], eager[0])
        for a, b in list(zip(outs, eager))[2:]:                            # (the embedding's are another kernel's, with atomics)
            assert torch.equal(a, b)


def test_another_stream():
    offsets, _, positions, T = batch()
    q, k, v = (randn(i, T, h, D) for i, h in enumerate((H, HK, HK)))
    want = sdgp.sdgp_attention(q, k, v, offsets)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x = q * 1.0
        got = sdgp.sdgp_attention(x, k, v, offsets)
        loss = sdgp.sdgp_policy_loss(got[1][:, 0].contiguous(), got[1][:, 1].contiguous(), got[1][:, 2].contiguous())[0]
    side.synchronize()
    assert all(map(torch.equal, got, want)) and math.isfinite(loss.item())


def test_gradients_that_are_not_asked_for():
    """k alone, a loss without gradient for its other outputs, expanded gradients."""
    offsets, _, positions, T = batch()
    freqs = torch.ones(D // 2, device="cuda")
    q, k = randn(0, T, H, D).requires_grad_(), randn(1, T, HK, D).requires_grad_()
    a, b = ag.sdgp_rotary(q, k, positions, freqs)
    assert torch.autograd.grad(b.sum(), k, retain_graph=True)[0].shape == k.shape
    assert torch.autograd.grad(a.sum(), q)[0].shape == q.shape
    o = ag.sdgp_attention(q.detach(), k, q.detach()[:, :HK].contiguous(), offsets)
    assert bool(torch.autograd.grad(o.sum(), k)[0].isfinite().all())
    logp = randn(3, T).requires_grad_()
    loss, kl, clipped = ag.sdgp_policy_loss(logp, logp.detach(), randn(4, T), None, None, offsets)
    assert not kl.requires_grad and not clipped.requires_grad and loss.requires_grad


def test_losses_that_are_written_to():
    """loss /= n, and sums of what is reported: outputs are tensors of their own, and gradients scale with them."""
    offsets, _, _, T = batch()
    logp, old, adv = randn(3, T).requires_grad_(), randn(3, T), randn(4, len(LENS))
    for call in (lambda: ag.sdgp_policy_loss(logp, old, adv, old, None, offsets, kl=0.1), lambda: ag.sdgp_preference_loss(logp, old, None, offsets)):
        loss, *reported = call()
        whole = torch.autograd.grad(loss, logp)[0]
        loss, *reported = call()
        kept = loss.item()
        for r in reported:
            r += 1
        loss /= 4
        loss += 1
        assert math.isclose(loss.item(), kept / 4 + 1, rel_tol=1e-6)
        assert torch.equal(torch.autograd.grad(loss, logp)[0], whole / 4)      # a power of two: exact

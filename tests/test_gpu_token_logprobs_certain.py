"""The gradient at a token that is almost certain: g (1 - p) with p next to 1.

Bound: what ln p itself is off by, as the forward call gives it, plus six roundings (e = 2^-24) of the element's own size (the
exponential minus one, two products, the scale, storing in fp32, the sizes' own roundings):
    |d - exact| <= scale |g| (|logp - exact logp| + 6 e (1 - p)).
A difference 1 - p of the rounded p is off by up to e/2 to 2 e of 1, far above that where 1 - p is small."""
import numpy as np
import pytest
import torch

import paper_2202_00774_amd as sdgp

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


def rows_of(V, seed, rows=400):
    """Logits whose first token of a random place has 1 - p between 1e-1 and 1e-6."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, V)).astype(np.float32)
    tokens = rng.integers(0, V, rows)
    rest = rng.uniform(1, 6, rows) * np.log(10)
    x[np.arange(rows), tokens] = -np.inf
    x[np.arange(rows), tokens] = np.log(np.exp(x.astype(np.float64)).sum(1)) + rest
    return x, tokens


@pytest.mark.parametrize("V", [2, 41, 64, 300, 1000, 4099, 20011])
def test_no_further_off_than_the_log_probability(V):
    x, tokens = rows_of(V, V)
    g = np.random.default_rng(1).normal(size=len(x)).astype(np.float32)
    for scale in (1.0, 0.75):
        z = scale * (x.astype(np.float64) - x.max(1, keepdims=True).astype(np.float64))
        others = np.exp(z)
        at = np.arange(len(x)), tokens
        top = others[at].copy()
        others[at] = 0.0
        r = others.sum(1) / top                                    # sum of the others over the token: p = 1 / (1 + r)
        lnp, rest = -np.log1p(r), r / (1 + r)
        gx, gt, gg = torch.from_numpy(x).cuda(), torch.from_numpy(tokens).cuda(), torch.from_numpy(g).cuda()
        logp, entropy, _, _, stats = sdgp.sdgp_token_logprobs(gx, gt, scale=scale)
        for h in (None, torch.zeros_like(gg)):
            d = sdgp.sdgp_token_logprobs_bwd(gx, gt, stats, entropy, gg, h, scale=scale).double().cpu().numpy()[at]
            exact = scale * g * rest
            off = np.abs(d - exact) - scale * np.abs(g) * (np.abs(logp.double().cpu().numpy() - lnp) + 6 * E * rest)
            assert (off <= 0).all(), (V, scale, off.max(), np.argmax(off))


def test_a_token_in_the_last_vectors_padding_writes_nothing_behind_the_row():
    """Tokens just outside an odd vocabulary, in rows cut out of wider ones: NaN in the row, nothing behind it."""
    for dtype in (torch.float32, torch.bfloat16):
        for V in (5, 41, 301, 1001, 9003):
            x = torch.randn(6, V + 16, device="cuda").to(dtype)[:, :V]
            tokens = torch.arange(V, V + 6, device="cuda")
            _, entropy, _, _, stats = sdgp.sdgp_token_logprobs(x, tokens)
            wide = torch.full((6, V + 16), 7.0, device="cuda", dtype=dtype)
            sdgp.sdgp_token_logprobs_bwd(x, tokens, stats, entropy, torch.ones(6, device="cuda"), torch.ones(6, device="cuda"), out=wide[:, :V])
            assert torch.isnan(wide[:, :V]).all() and (wide[:, V:] == 7).all()

"""The step lr / bc1 * m / (sqrt(v) / sqrt(bc2) + eps) itself, for either kind of state.

From parameters of zero with eps = 0 a step is four fp32 operations behind m and v, one rounding each (root, product, quotient,
product), and the library's first step is m = (1 - beta1) g, v = (1 - beta2) g^2: numpy's fp32 gives the same bits.
"""
import numpy as np
import pytest
import torch

from paper_2202_00774_amd.optim import AdamW

pytestmark = pytest.mark.gpu
F = np.float32


def first_step(g, bits, eps, lr=3e-3, betas=(0.85, 0.995)):
    p = torch.zeros(len(g), device="cuda")
    AdamW([p], lr=lr, betas=betas, eps=eps, weight_decay=0.1, state_bits=bits).step([torch.from_numpy(g).cuda()])
    m, v = g * F(1 - betas[0]), (g * g) * F(1 - betas[1])
    with np.errstate(divide="ignore", invalid="ignore"):
        den = (np.sqrt(v) * F(1 / np.sqrt(1 - betas[1]))).astype(np.float64) + np.float64(F(eps))
        want = -(F(lr / (1 - betas[0])) * (m / den.astype(F)))
    assert want.dtype == F
    return p.cpu().numpy(), want


@pytest.mark.parametrize("bits", [8, 32])
def test_every_bit_of_a_step(bits):
    rng = np.random.default_rng(bits)
    g = (rng.normal(size=20000) * 10.0 ** rng.uniform(-8, 8, 20000)).astype(F)
    got, want = first_step(g, bits, 0.0)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_denominator_of_zero_and_below_the_normal_numbers(bits):
    g = np.array([0.0, 1.0, -2.0, 0.0, 1e-30, -1e-25], F)       # the squares of the last two are 0
    got, want = first_step(g, bits, 0.0)
    assert np.array_equal(np.isnan(want), [True, False, False, True, False, False]) and np.isinf(want[4:]).all()
    assert np.array_equal(got, want, equal_nan=True)
    got, want = first_step(g, bits, 1e-40)
    assert np.isfinite(want).all() and abs(want[4]) > 1e6
    assert np.array_equal(got, want)

"""Block norms with values that are not finite, or whose squares are not."""
import pytest
import torch

import paper_2202_00774_amd as sdgp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [24, 130, 264, 500])
@pytest.mark.parametrize("rows,gates", [(4100, 2050), (2050, 2050), (1027, 1027), (6, 3), (4, 1)])
def test_an_infinite_gate(rows, gates, D, dtype):
    """dL/dw_post is the sum of dY gate a: where one gate is infinite and its dY a is not 0, infinite, of that product's sign.  Every
    other column and gate stays finite.  (Without the norm behind dY is dy, so the infinity stays in its column; y's is not read.)"""
    torch.manual_seed(D)
    x, u, dy = (torch.randn(rows, D, device="cuda").to(dtype) for _ in range(3))
    gate, w = torch.randn(gates, D, device="cuda").to(dtype), torch.ones(D, device="cuda")
    hit, col, per = gates - 1 - (gates - 1) % 2 if gates > 1 else 0, 3, rows // gates
    y, _, stats = sdgp.sdgp_block_norm(x, u, gate, w, None, pre=False)
    gate[hit, col] = float("inf")
    dx, du, dgate, dw_post, _ = sdgp.sdgp_block_norm_bwd(dy, None, y, stats, u, gate, w, None)
    mine = slice(hit * per, (hit + 1) * per)
    sign = torch.sign((dy[mine, col].double() * u[mine, col].double()).sum())          # the rows' factors are near to each other
    if (torch.sign(dy[mine, col].float() * u[mine, col].float()) == sign).all():
        assert dw_post[col] == sign * float("inf")
    else:
        assert not torch.isfinite(dw_post[col])
    keep = torch.arange(D, device="cuda") != col
    assert torch.isfinite(dw_post[keep]).all() and torch.isfinite(dgate).all() and torch.isfinite(dx).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_squares_beyond_the_range(dtype):
    """The sum of a row's squares is fp32: where it is not finite the factor is 0, and the gradient through the norm with it."""
    torch.manual_seed(0)
    x, u = (torch.randn(3, 264, device="cuda").to(dtype) for _ in range(2))
    u[1] = 1e20
    x[2] = -3e20
    y, h, stats = sdgp.sdgp_block_norm(x, u)
    assert torch.equal(y[1], x[1]) and stats[0, 1] == 0 and stats[1, 2] == 0 and (h[2] == 0).all() and torch.isfinite(h).all()
    dx, du, *_ = sdgp.sdgp_block_norm_bwd(x, u, y, stats, u)
    assert (du[1] == 0).all() and torch.equal(dx[2], x[2]) and torch.isfinite(dx).all() and torch.isfinite(du).all()

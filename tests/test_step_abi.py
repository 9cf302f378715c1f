"""Argument checks of the operators around the pruned layers, at the C boundary and in the binding, without a GPU."""
import ctypes

import pytest
import torch

import paper_2202_00774_amd as sdgp
from paper_2202_00774_amd import autograd, binding
from paper_2202_00774_amd.optim import AdamW

OK, E_NULL, E_SHAPE, E_DTYPE, E_WS, E_VALUE = 0, -1, -3, -4, -6, -8
P, P2, ODD = ctypes.c_void_p(16), ctypes.c_void_p(18), ctypes.c_void_p(17)       # never dereferenced
BAD = ctypes.c_size_t(-1).value
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def test_value_status(lib):
    assert binding.status_string(-8) not in ("unknown status", "") and binding.status_string(-9) == "unknown status"


def test_token_logprobs_argument_errors(lib):
    def call(logits=P, ld=16, tokens=P, bits=64, logp=P, entropy=P, top_logp=P, top_ids=P, stats=P, rows=2, V=16, dt=1, top=4, scale=1.0,
             ws=P, ws_bytes=1 << 30):
        return lib.sdgp_token_logprobs(logits, ld, tokens, bits, logp, entropy, top_logp, top_ids, stats, rows, V, dt, top, scale, ws, ws_bytes, None)

    assert call(dt=2) == E_DTYPE and call(bits=16) == E_DTYPE
    assert call(rows=-1) == E_SHAPE and call(V=0) == E_SHAPE and call(ld=15) == E_SHAPE
    assert call(V=2**30 + 1, ld=2**30 + 1) == E_SHAPE and call(rows=2**39, ld=16) == E_SHAPE
    assert call(top=-1) == E_SHAPE and call(top=65, V=100, ld=100) == E_SHAPE and call(top=17) == E_SHAPE
    for scale in (0.0, -1.0, INF, NAN):
        assert call(scale=scale) == E_VALUE
    assert call(logits=None) == E_NULL and call(entropy=None) == E_NULL and call(stats=None) == E_NULL
    assert call(tokens=None) == E_NULL                       # logp of which tokens?
    assert call(top_ids=None) == E_NULL and call(top_logp=None) == E_NULL
    assert call(logits=ODD) == E_SHAPE and call(logits=P2, dt=0) == E_SHAPE and call(tokens=P2) == E_SHAPE
    assert call(rows=0, logits=None) == OK
    assert lib.sdgp_token_logprobs_workspace(2, 16, 3, 0) == BAD and lib.sdgp_token_logprobs_workspace(2, 16, 1, 17) == BAD
    need = lib.sdgp_token_logprobs_workspace(1, 1 << 20, 1, 8)
    assert need != BAD
    if need:
        assert call(rows=1, V=1 << 20, ld=1 << 20, top=8, ws=None) == E_WS and call(rows=1, V=1 << 20, ld=1 << 20, top=8, ws_bytes=need - 1) == E_WS
        assert call(rows=1, V=1 << 20, ld=1 << 20, top=8, ws=ctypes.c_void_p(24)) == E_WS


def test_token_logprobs_bwd_argument_errors(lib):
    def call(logits=P, ld=16, tokens=P, bits=64, stats=P, entropy=P, g=P, h=P, out=P, ld_out=16, rows=2, V=16, dt=1, scale=1.0):
        return lib.sdgp_token_logprobs_bwd(logits, ld, tokens, bits, stats, entropy, g, h, out, ld_out, rows, V, dt, scale, None)

    assert call(dt=-1) == E_DTYPE and call(bits=8) == E_DTYPE
    assert call(V=0) == E_SHAPE and call(ld=15) == E_SHAPE and call(ld_out=15) == E_SHAPE and call(rows=-1) == E_SHAPE
    assert call(scale=0.0) == E_VALUE and call(scale=NAN) == E_VALUE
    assert call(logits=None) == E_NULL and call(stats=None) == E_NULL and call(out=None) == E_NULL
    assert call(tokens=None) == E_NULL and call(entropy=None) == E_NULL and call(g=None, h=None) == E_NULL
    assert call(out=ODD) == E_SHAPE and call(tokens=P2) == E_SHAPE
    assert call(rows=0) == OK


def test_block_norm_argument_errors(lib):
    def call(x=P, u=P, gate=P, w_post=P, w_pre=P, y=P, h=P, stats=P, rows=6, D=8, groups=2, dt=1, wdt=0, rs=1.0, eps=1e-6):
        return lib.sdgp_block_norm(x, u, gate, w_post, w_pre, y, h, stats, rows, D, groups, dt, wdt, rs, eps, None)

    assert call(dt=4) == E_DTYPE and call(wdt=4) == E_DTYPE
    assert call(rows=-1) == E_SHAPE and call(D=0) == E_SHAPE and call(groups=4) == E_SHAPE and call(groups=-1) == E_SHAPE
    assert call(rs=INF) == E_VALUE and call(eps=-1.0) == E_VALUE and call(eps=NAN) == E_VALUE
    assert call(x=None) == E_NULL and call(stats=None) == E_NULL and call(y=None) == E_NULL
    assert call(u=None) == E_NULL                            # gate, w_post and y without a block
    assert call(gate=None) == E_NULL and call(groups=0) == E_NULL
    assert call(h=None) == E_NULL                            # w_pre without its norm
    assert call(u=None, gate=None, groups=0, w_post=None, y=None, h=None, w_pre=None) == E_NULL
    assert call(x=ODD) == E_SHAPE and call(w_pre=P2) == E_SHAPE and call(gate=ODD) == E_SHAPE
    assert call(rows=0) == OK


def test_block_norm_bwd_argument_errors(lib):
    def call(dy=P, dh=P, y=P, u=P, gate=P, w_post=P, w_pre=P, stats=P, dx=P, du=P, dgate=P, dw_post=P, dw_pre=P, rows=6, D=8, groups=2,
             dt=1, wdt=0, rs=1.0, ws=P, ws_bytes=1 << 30):
        return lib.sdgp_block_norm_bwd(dy, dh, y, u, gate, w_post, w_pre, stats, dx, du, dgate, dw_post, dw_pre, rows, D, groups, dt, wdt,
                                       rs, ws, ws_bytes, None)

    assert call(dt=4) == E_DTYPE and call(wdt=-1) == E_DTYPE
    assert call(groups=5) == E_SHAPE and call(D=0) == E_SHAPE
    assert call(rs=NAN) == E_VALUE
    for name in ("y", "u", "gate", "w_post", "w_pre", "stats", "dx", "du", "dgate", "dw_post", "dw_pre", "dh"):
        assert call(**{name: None}) == E_NULL, name
    assert call(dy=None, dh=None, w_pre=None, dw_pre=None) == E_NULL
    assert call(du=ODD) == E_SHAPE and call(w_post=P2) == E_SHAPE
    need = lib.sdgp_block_norm_bwd_workspace(6, 8, 2, 1)
    assert need not in (0, BAD)
    assert call(ws=None) == E_WS and call(ws_bytes=need - 1) == E_WS and call(ws=ctypes.c_void_p(20)) == E_WS
    assert lib.sdgp_block_norm_bwd_workspace(6, 8, 4, 1) == BAD and lib.sdgp_block_norm_bwd_workspace(0, 8, 0, 1) == 0
    assert call(rows=0, groups=0, gate=None, dgate=None, w_post=None, dw_post=None, w_pre=None, dw_pre=None) == OK


def adamw(lib, n=(300,), count=None, p=16, g=16, m=16, v=16, ms=16, vs=16, copies=None, pdt=0, gdt=0, bits=32, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8,
          wd=0.0, step=1, arrays=True):
    k = len(n)
    ptrs = lambda x: None if x is None else (ctypes.c_void_p * k)(*([x or None] * k))  # noqa: E731
    return lib.sdgp_adamw_step(k if count is None else count, ptrs(p) if arrays else None, ptrs(g), ptrs(m), ptrs(v), ptrs(ms), ptrs(vs), ptrs(copies),
                               (ctypes.c_int64 * k)(*n), pdt, gdt, bits, lr, b1, b2, eps, wd, step, None, 0, None)


def test_adamw_argument_errors(lib):
    assert adamw(lib, pdt=2) == E_DTYPE and adamw(lib, gdt=-1) == E_DTYPE and adamw(lib, bits=16) == E_DTYPE
    assert adamw(lib, pdt=1, copies=16) == E_DTYPE           # a bf16 parameter is its own copy
    assert adamw(lib, n=(-1,)) == E_SHAPE and adamw(lib, n=(2**41,)) == E_SHAPE and adamw(lib, n=(2**40, 2**40)) == E_SHAPE
    assert adamw(lib, count=-1) == E_SHAPE
    for bad in (dict(lr=-1.0), dict(lr=NAN), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=NAN), dict(eps=-1.0), dict(eps=INF), dict(wd=-1.0), dict(step=0)):
        assert adamw(lib, **bad) == E_VALUE, bad
    assert adamw(lib, arrays=False) == E_NULL
    for name in ("p", "g", "m", "v"):
        assert adamw(lib, **{name: 0}) == E_NULL, name
    assert adamw(lib, bits=8, ms=None) == E_NULL and adamw(lib, bits=8, vs=0) == E_NULL and adamw(lib, copies=0) == E_NULL
    assert adamw(lib, p=18) == E_SHAPE and adamw(lib, g=17, gdt=1) == E_SHAPE and adamw(lib, m=18) == E_SHAPE and adamw(lib, copies=17) == E_SHAPE
    assert adamw(lib, bits=8, ms=18) == E_SHAPE
    assert adamw(lib, count=0, arrays=False) == OK
    assert adamw(lib, n=(0, 0), p=0, g=0) == OK              # nothing in them


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU"):
        sdgp.sdgp_token_logprobs(x, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError, match="GPU"):
        sdgp.sdgp_block_norm(x)
    with pytest.raises(ValueError, match="GPU"):
        AdamW([x])
    with pytest.raises(ValueError):
        AdamW([], state_bits=4)


def test_rows_may_be_strided_but_evenly():
    cuda_like = type("T", (torch.Tensor,), {"is_cuda": property(lambda self: True)})

    def stride(t):
        return binding._row_stride(t.as_subclass(cuda_like), "t")

    wide = torch.zeros(6, 40)
    assert stride(wide) == 40 and stride(wide[:, 3:20]) == 40 and stride(wide[::2, :7]) == 80
    assert stride(wide.view(2, 3, 40)[..., :9]) == 40 and stride(wide.view(2, 3, 40)[:, :1, :9]) == 120
    assert stride(wide[:1, :5]) == 5 and stride(wide[0, :5]) == 5 and stride(torch.zeros(1, 1, 40)[..., :4]) == 4
    for bad in (wide.t(), wide[:, ::2], wide[:1].expand(6, 40), wide.view(2, 3, 40)[:, :2], torch.zeros(4, 8).as_strided((4, 8), (4, 1))):
        with pytest.raises(ValueError):
            stride(bad)

"""The operators around the pruned layers take tensors of one GPU.  Without a GPU: tensors that say they are on one, and a
library that must not be called with others."""
import types

import pytest
import torch

import paper_2202_00774_amd as sdgp
from paper_2202_00774_amd import binding


class OnGpu(torch.Tensor):
    gpu = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.gpu


def on(gpu, *shape, dtype=torch.float32):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)
    t.gpu = gpu
    return t


@pytest.fixture
def calls(monkeypatch):
    seen = []
    names = ("sdgp_token_logprobs", "sdgp_token_logprobs_bwd", "sdgp_block_norm", "sdgp_block_norm_bwd")
    lib = types.SimpleNamespace(**{n: lambda *a, n=n: seen.append(n) or 0 for n in names})
    monkeypatch.setattr(binding, "load", lambda: lib)
    monkeypatch.setattr(binding, "_need", lambda *a: 64)
    monkeypatch.setattr(binding, "_stream", lambda t: 0)
    return seen


def each(call, args, calls):
    """call(**args) goes through; with any one of the tensors elsewhere, on another GPU or on the host, it is refused."""
    call(**args)
    assert len(calls) == 1
    for name, t in args.items():
        for gpu in (1, -1):
            other = on(gpu, *t.shape, dtype=t.dtype)
            with pytest.raises(ValueError, match="GPU"):
                call(**{**args, name: other})
    assert len(calls) == 1


def test_token_logprobs(calls):
    x = on(0, 4, 9)
    each(lambda **k: sdgp.sdgp_token_logprobs(x, **k), {"tokens": on(0, 4, dtype=torch.int64), "workspace": on(0, 64, dtype=torch.uint8)}, calls)


def test_token_logprobs_gradient(calls):
    x = on(0, 4, 9)
    each(lambda **k: sdgp.sdgp_token_logprobs_bwd(x, **k),
         {"tokens": on(0, 4, dtype=torch.int32), "stats": on(0, 4, 2), "entropy": on(0, 4), "g_logp": on(0, 4), "g_entropy": on(0, 4), "out": on(0, 4, 9)}, calls)


def test_block_norm(calls):
    x = on(0, 4, 8)
    each(lambda **k: sdgp.sdgp_block_norm(x, **k), {"u": on(0, 4, 8), "gate": on(0, 2, 8), "w_post": on(0, 8), "w_pre": on(0, 8)}, calls)


def test_block_norm_gradient(calls):
    y = on(0, 4, 8)
    each(lambda **k: sdgp.sdgp_block_norm_bwd(y=y, **k),
         {"dy": on(0, 4, 8), "dh": on(0, 4, 8), "stats": on(0, 2, 4), "u": on(0, 4, 8), "gate": on(0, 2, 8), "w_post": on(0, 8), "w_pre": on(0, 8),
          "workspace": on(0, 64, dtype=torch.uint8)}, calls)


def test_a_workspace_holds_its_bytes(calls):
    """An expanded one counts them without having them."""
    x, few = on(0, 4, 9), on(0, 1, dtype=torch.uint8)
    with pytest.raises(ValueError, match="contiguous"):
        sdgp.sdgp_token_logprobs(x, None, workspace=few.expand(64))

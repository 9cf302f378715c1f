"""AdamW.step with and without torch's call that recognises a list of tensors: what it does not recognise is checked in Python, and
the same lists are taken and refused.  Without a GPU: the library is a stand-in, tensors count as the GPU's."""
import types

import pytest
import torch

from paper_2202_00774_amd import binding, optim

BF16 = torch.bfloat16


@pytest.mark.parametrize("guards", [True, False])
def test_the_same_lists_are_taken_and_refused(guards, monkeypatch):
    calls = []
    monkeypatch.setattr(binding, "load", lambda: types.SimpleNamespace(sdgp_adamw_step=lambda *a: calls.append(list(a[2])) or 0))
    monkeypatch.setattr(binding, "_stream", lambda t: 0)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    if not guards:
        monkeypatch.setattr(optim, "_guards", None)
    params, copies = [torch.zeros(6, 6), torch.zeros(5), torch.zeros(0)], [torch.zeros(6, 6, dtype=BF16), torch.zeros(5, dtype=BF16), torch.zeros(0, dtype=BF16)]
    opt = optim.AdamW(params, copies=copies)

    def grads(dtype=torch.float32):
        return [torch.ones(p.shape, dtype=dtype) for p in params]

    for g in (grads(), grads(), grads(BF16), grads()):          # new tensors every time, and another dtype
        opt.step(g)
        assert calls[-1][:2] == [t.data_ptr() for t in g[:2]]
    taken = len(calls)
    bad = [grads() for _ in range(6)]
    bad[0][0] = torch.ones(6, 6).t()
    bad[1][0] = torch.ones(6, 7)[:, :6]
    bad[2][1] = torch.ones(5, dtype=BF16)
    bad[3][1] = torch.ones(4)
    bad[4][1] = None
    bad[5] = bad[5][:2]
    for g in bad:
        with pytest.raises(ValueError):
            opt.step(g)
    for t in (params[0], copies[0]):
        t.data = t.data.t()
        with pytest.raises(ValueError):
            opt.step(grads())
        t.data = t.data.t()
    assert len(calls) == opt.steps == taken
    g = grads()
    g[1] = g[0].view(-1)[:5]                                    # gradients may share memory: they are only read
    opt.step(g)
    with torch.inference_mode():
        opt.step(g)
    opt.step(grads())
    assert len(calls) == opt.steps == taken + 3

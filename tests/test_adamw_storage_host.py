"""What AdamW.step looks at before it hands addresses to the library, without a GPU: the library is a stand-in that records
the call, and tensors count as the GPU's."""
import types

import pytest
import torch

from paper_2202_00774_amd import binding
from paper_2202_00774_amd.optim import AdamW

BF16 = torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    """The library's calls, as lists of addresses: (params, grads, exp_avg, exp_avg_sq, scales, scales, copies)."""
    seen = []

    def step(count, *rest):
        seen.append([None if a is None else list(a) for a in rest[:7]])
        return 0

    monkeypatch.setattr(binding, "load", lambda: types.SimpleNamespace(sdgp_adamw_step=step))
    monkeypatch.setattr(binding, "_stream", lambda t: 0)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    return seen


def optimizer(calls, *shapes, **kw):
    """Params, their gradients and an optimizer that has made a step."""
    params, grads = [torch.zeros(s) for s in shapes], [torch.ones(s) for s in shapes]
    opt = AdamW(params, **kw)
    opt.step(grads)
    assert len(calls) == opt.steps == 1 and calls[0][0] == [p.data_ptr() for p in params]
    return params, grads, opt


def refused(opt, grads, calls):
    with pytest.raises(ValueError):
        opt.step(grads)
    assert len(calls) == opt.steps == 1


def test_other_strides_at_the_same_address(calls):
    (p, _), grads, opt = optimizer(calls, (6, 6), (5,))
    p.data = p.data.t()                                    # square: the shape is what it was
    refused(opt, grads, calls)


def test_another_dtype_at_the_same_address(calls):
    (p, _), grads, opt = optimizer(calls, (6, 6), (5,))
    p.data = torch.empty(0, dtype=BF16).set_(p.data.view(BF16).untyped_storage(), 0, (6, 6))
    assert p.dtype == BF16 and p.is_contiguous()
    refused(opt, grads, calls)


def test_another_size_at_the_same_address(calls):
    (p, _), grads, opt = optimizer(calls, (6, 6), (5,))
    p.data = p.data[:3]
    refused(opt, grads, calls)


def test_copies_too(calls):
    copy = torch.zeros(6, 6, dtype=BF16)
    (p,), grads, opt = optimizer(calls, (6, 6), copies=[copy])
    copy.data = copy.data.t()
    refused(opt, grads, calls)
    copy.data = torch.zeros(6, 6, dtype=BF16)              # whole again, somewhere else
    opt.step(grads)
    assert calls[1][6] == [copy.data_ptr()]


def test_params_that_moved_to_another_gpu(calls, monkeypatch):
    params, grads, opt = optimizer(calls, (6, 6), (5,))
    for p in params:
        p.data = p.data.clone()
    there = {t.data_ptr() for t in (*params, *grads)}
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: int(t.data_ptr() in there))
    refused(opt, grads, calls)                             # the states stayed


@pytest.mark.parametrize("bits", [8, 32])
def test_states_that_were_put_away_and_brought_back(calls, bits):
    """Whoever holds state() shares its storage, and may free it and allocate it again between steps."""
    _, grads, opt = optimizer(calls, (600,), (5,), state_bits=bits)
    held = opt.state()
    hold = []
    for tensors in held.values():
        for t in tensors:
            storage, was = t.untyped_storage(), t.data_ptr()
            size = storage.nbytes()
            storage.resize_(0)
            while t.data_ptr() in (0, was):
                hold.append(torch.empty(size, dtype=torch.uint8))
                storage.resize_(0), storage.resize_(size)
    opt.step(grads)
    for k, name in enumerate(held):
        assert calls[1][2 + k] == [t.data_ptr() for t in held[name]] != calls[0][2 + k]


def test_states_that_are_not_there(calls):
    _, grads, opt = optimizer(calls, (600,), (5,))
    storage = opt.state()["exp_avg"][0].untyped_storage()
    storage.resize_(0)
    refused(opt, grads, calls)
    storage.resize_(400)                                   # part of it
    refused(opt, grads, calls)
    storage.resize_(2400)
    opt.step(grads)
    assert calls[1][2][0] == opt.state()["exp_avg"][0].data_ptr()


def test_a_refusal_is_not_forgotten(calls, monkeypatch):
    """Storage that was freed can come back smaller at the address it had: the step after a refusal checks it all."""
    _, grads, opt = optimizer(calls, (600,), (5,))
    t = opt.state()["exp_avg"][0]
    storage, was, plain = t.untyped_storage(), t.data_ptr(), torch.Tensor.data_ptr
    storage.resize_(0)
    refused(opt, grads, calls)
    storage.resize_(400)
    there = plain(t)
    monkeypatch.setattr(torch.Tensor, "data_ptr", lambda x: was if plain(x) == there else plain(x))
    monkeypatch.setattr(opt, "_check_places", lambda: pytest.fail("looked at", pytrace=False))
    with pytest.raises(pytest.fail.Exception, match="looked at"):
        opt.step(grads)


def test_tensors_that_share_memory(calls):
    room = torch.zeros(1000)
    ok = AdamW([room[:300], room[300:301], room[301:301], room[301:]])       # side by side
    with pytest.raises(ValueError, match="share memory"):
        AdamW([room[:300], room[299:]])
    with pytest.raises(ValueError, match="share memory"):
        AdamW([room[:300], room[300:]], copies=[room.view(BF16)[1400:1700], torch.zeros(700, dtype=BF16)])
    same = [torch.zeros(300), torch.zeros(1), torch.zeros(0), torch.zeros(699)]
    with pytest.raises(ValueError, match="share memory"):
        AdamW(ok.params, state={"exp_avg": same, "exp_avg_sq": same})
    with pytest.raises(ValueError, match="share memory"):
        AdamW([room[:300]], state={"exp_avg": [room[200:500]], "exp_avg_sq": [torch.zeros(300)]})
    ok.step([torch.ones(p.shape) for p in ok.params])
    ok.params[1].data = room[500:501]                                        # into another one's place
    for _ in range(2):
        refused(ok, [torch.ones(p.shape) for p in ok.params], calls)
    ok.params[1].data = torch.zeros(1)
    ok.step([torch.ones(p.shape) for p in ok.params])
    assert len(calls) == 2

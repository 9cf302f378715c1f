"""Convolution weights as sdgp_conv2d reads them best: four dimensions, channels last.  A step goes element by element, so it
gives what it gives for the same weights as a contiguous [out, R, S, in] tensor, bit for bit."""
import pytest
import torch

from paper_2202_00774_amd.autograd import sdgp_conv2d
from paper_2202_00774_amd.optim import AdamW

pytestmark = pytest.mark.gpu
BF16, LAST = torch.bfloat16, torch.channels_last
SHAPES = [(8, 5, 3, 3), (7,), (64, 16, 3, 3), (16, 8, 1, 1), (4, 1, 3, 3), (1, 6, 2, 5)]


def krsc(t):
    """A [out, R, S, in] tensor of its own.  (The permuted view of a channels-last tensor is contiguous: contiguous() would share it.)"""
    return (t.permute(0, 2, 3, 1) if t.dim() == 4 else t).clone(memory_format=torch.contiguous_format)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype,copies", [(torch.float32, True), (BF16, False)])
def test_the_same_bits_as_contiguous_weights(bits, dtype, copies):
    g = torch.Generator(device="cuda")
    g.manual_seed(bits)
    rnd = lambda: [torch.randn(s, device="cuda", generator=g).to(dtype) for s in SHAPES]  # noqa: E731
    last = [t.contiguous(memory_format=LAST) if t.dim() == 4 else t for t in rnd()]
    flat = [krsc(t) for t in last]
    low = [[torch.empty_like(t, dtype=BF16) for t in ts] for ts in (last, flat)] if copies else [None, None]
    assert last[0].stride() == (45, 1, 15, 5)
    opts = [AdamW(ts, state_bits=bits, copies=c, seed=3) for ts, c in zip((last, flat), low)]
    for _ in range(3):
        grads = rnd()
        opts[0].step([t.contiguous(memory_format=LAST) if t.dim() == 4 else t for t in grads])
        opts[1].step([krsc(t) for t in grads])
    state = [o.state() for o in opts]
    assert state[0]["exp_avg"][0].stride() == (45, 1, 15, 5)
    pairs = [(last, flat), *((state[0][k], state[1][k]) for k in ("exp_avg", "exp_avg_sq"))] + ([(low[0], low[1])] if copies else [])
    for a, b in pairs:
        for p, q in zip(a, b):
            assert torch.equal(krsc(p.float()), q.float())
    twin = AdamW([t.clone() for t in last], state_bits=bits, seed=3, state=state[0], steps=3)      # goes on from such a state
    assert twin.state()["exp_avg"][0].data_ptr() == state[0]["exp_avg"][0].data_ptr()


def test_a_convolution_is_trained():
    torch.manual_seed(0)
    w = torch.nn.Parameter(torch.randn(16, 8, 3, 3, device="cuda", dtype=BF16).contiguous(memory_format=LAST))
    x = torch.randn(2, 8, 9, 9, device="cuda", dtype=BF16).contiguous(memory_format=LAST)
    opt = AdamW([w], lr=0.01)
    before, size = w.detach().clone(), []
    for step in range(6):
        w.grad = None
        loss = sdgp_conv2d(x, w, 1, 1, seed=step).float().square().mean()
        loss.backward()
        opt.step()
        size.append(loss.item())
    assert not torch.equal(before, w) and size[-1] < size[0]


def test_layouts_that_do_not_agree_are_refused():
    w = torch.zeros(8, 5, 3, 3, device="cuda").contiguous(memory_format=LAST)
    opt = AdamW([w])
    with pytest.raises(ValueError):
        opt.step([torch.zeros(8, 5, 3, 3, device="cuda")])
    with pytest.raises(ValueError):
        AdamW([w], copies=[torch.zeros(8, 5, 3, 3, device="cuda", dtype=BF16)])
    with pytest.raises(ValueError):
        AdamW([w], state={k: [torch.zeros(8, 5, 3, 3, device="cuda")] for k in ("exp_avg", "exp_avg_sq")})
    with pytest.raises(ValueError):
        AdamW([torch.zeros(8, 5, 3, 3, device="cuda").transpose(0, 2)])
    w.data = torch.zeros(8, 5, 3, 3, device="cuda")                 # the states stay as they are
    with pytest.raises(ValueError):
        opt.step([torch.zeros(8, 5, 3, 3, device="cuda")])
    assert opt.steps == 0

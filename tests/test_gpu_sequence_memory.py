"""What the operators on packed sequences write to, where offsets and lengths are wrong: their outputs and workspace and nothing
around them, and none of their inputs."""
import ctypes

import pytest
import torch

from paper_2202_00774_amd import binding

pytestmark = pytest.mark.gpu
MARGIN, PATTERN = 1 << 16, 0xA5


class Guarded:
    """Tensors in the middle of larger buffers, with a pattern on both sides (and within, for outputs)."""

    def __init__(self):
        self.held = []

    def _take(self, nbytes):
        buffer = torch.full((MARGIN + nbytes + MARGIN,), PATTERN, dtype=torch.uint8, device="cuda")
        return buffer, buffer[MARGIN:MARGIN + nbytes]

    def output(self, *shape, dtype):
        buffer, middle = self._take(torch.empty(shape, dtype=dtype, device="meta").nbytes)
        self.held.append((buffer, middle, None))
        return middle.view(dtype).view(shape)

    def input(self, t):
        buffer, middle = self._take(t.nbytes)
        middle.copy_(t.contiguous().view(-1).view(torch.uint8))
        self.held.append((buffer, middle, middle.clone()))
        return middle.view(t.dtype).view(t.shape)

    def check(self):
        torch.cuda.synchronize()
        for buffer, middle, content in self.held:
            assert bool((buffer[:MARGIN] == PATTERN).all()) and bool((buffer[MARGIN + middle.numel():] == PATTERN).all())
            assert content is None or torch.equal(middle, content)


def randn(seed, *shape, dtype=torch.float32):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def call(name, *args):
    args = [None if a is None else binding._ptr(a) if isinstance(a, torch.Tensor) else a for a in args]
    assert getattr(binding.load(), name)(*args, torch.cuda.current_stream().cuda_stream) == 0


def attention(bad_q, bad_k, lengths, T, Tk, H, Hk, D, dtype, causal, backward=True):
    g, S = Guarded(), (len(lengths) if lengths else len(bad_q) - 1)
    q, k, v, do = (g.input(randn(i, t, h, D, dtype=dtype)) for i, (t, h) in enumerate(((T, H), (Tk, Hk), (Tk, Hk), (T, H))))
    off_q, off_k, filled = (None if x is None else g.input(ints(x)) for x in (bad_q, bad_k, lengths))
    strides, code = (ctypes.c_int64 * 6)(H * D, D, Hk * D, D, Hk * D, D), binding._dtype_code(q)
    sizes = (T, Tk, H, Hk, D, code)
    o, lse = g.output(T, H, D, dtype=dtype), g.output(T, H, dtype=torch.float32)
    need = binding._need("sdgp_attention_workspace", S, *sizes)
    ws = g.output(need, dtype=torch.uint8)
    call("sdgp_attention", q, k, v, strides, off_q, off_k, filled, S, o, lse, *sizes, int(causal), 0.1, ws if need else None, need)
    g.check()
    if not backward:
        return
    need = binding._need("sdgp_attention_bwd_workspace", S, *sizes)
    ws, dq, dk, dv = g.output(need, dtype=torch.uint8), *(g.output(*t.shape, dtype=dtype) for t in (q, k, v))
    call("sdgp_attention_bwd", do, q, k, v, o, lse, strides, off_q, off_k, S, dq, dk, dv, *sizes, int(causal), 0.1, ws, need)
    g.check()


BAD = [[0, 90, 50, 100], [-5, 30, 60, 100], [0, 50, 1000, 2000000000], [100, 50, 20, 0], [-2000000000, -1, -1, 101], [7, 7, 7, 7]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("D", [64, 33])
def test_attention_with_wrong_offsets(bad, D, causal, dtype):
    attention(bad, bad, None, 100, 100, 4, 2, D, dtype, causal)
    attention(bad, BAD[0], None, 100, 90, 4, 2, D, dtype, causal)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale_of", [[0, 1700, 900, 2000], [-5, 2500, -1, 700], [2000, 1000, 500, 0]])
def test_attention_with_wrong_offsets_in_larger_plans(scale_of, dtype):
    """Tiles in the order of their work, and keys in parts."""
    attention(scale_of, scale_of, None, 2000, 2000, 64, 32, 24, dtype, True)
    attention([0, 70, 30, 100], [2 * x for x in scale_of], None, 100, 4000, 2, 1, 64, dtype, True)
    attention(scale_of, scale_of, None, 2000, 2000, 4, 1, 33, dtype, True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [128, 33])
def test_attention_with_wrong_lengths(D, dtype):
    attention(None, None, [-1, 0, 2000000000, -2000000000, 700, 701], 6, 6 * 700, 8, 2, D, dtype, True, backward=False)


@pytest.mark.parametrize("T, bad", [(1000, [0, 500, 200, 700, 600]), (1000, [-10, 300, 300, 300, 9000]), (1000, [900, 100, 50, 20, 0]),
                                    (30000, [0, 25000, 100, 2000000000, -2000000000]), (30000, [-2000000000, 2000000000, -5, 30001, 30000])])
@pytest.mark.parametrize("each", [True, False])
def test_losses_with_wrong_offsets(T, bad, each):
    g, S = Guarded(), len(bad) - 1
    logp, old, ref, adv, one = (g.input(randn(i, n)) for i, n in enumerate((T, T, T, T if each else S, 1)))
    mask, offsets = g.input((randn(9, T) > 0).to(torch.uint8)), g.input(ints(bad))
    need = binding._need("sdgp_sequence_loss_workspace", T, S)
    f32 = {"dtype": torch.float32}
    ws, out, weights, dlogp = g.output(need, dtype=torch.uint8), g.output(3, **f32), g.output(S, **f32), g.output(T, **f32)
    policy = (logp, old, ref, adv, int(each), mask, offsets, S, T, 0.2, 0.2, 0.1)
    for by_sequence in (0, 1):
        call("sdgp_policy_loss", *policy, by_sequence, out, weights, ws, need)
        call("sdgp_policy_loss_bwd", one, weights, *policy, dlogp)
        g.check()
    loss, margins = g.output(1, **f32), g.output(S // 2, **f32)
    call("sdgp_preference_loss", logp, ref, mask, offsets, S, T, 0.1, 0.0, 0.1, 1, loss, margins, weights, ws, need)
    call("sdgp_preference_loss_bwd", one, weights, mask, offsets, S, T, dlogp)
    g.check()

"""Attention of packed sequences, its gradients and its form for caches, against 64 bits."""
import math

import pytest
import torch

import paper_2202_00774_amd as sdgp
from attention_reference import attention, check, spans_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def randn(seed, *shape, dtype=F32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


def offsets_of(lens, first=0):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def packed(lens_q, lens_k, dtype, H, Hk, D, causal, first=0, behind=0, seed=0):
    """Inputs as a layer leaves them, cut out of one tensor where the lengths are the same; checked forward and backward."""
    Tq, Tk = first + sum(lens_q) + behind, first + sum(lens_k) + behind
    if lens_q == lens_k:
        q, k, v = randn(seed, Tq, H + 2 * Hk, D, dtype=dtype).split((H, Hk, Hk), 1)
        off_q, off_k = offsets_of(lens_q, first), None
    else:
        q, k, v = randn(seed, Tq, H, D, dtype=dtype), *randn(seed + 1, Tk, 2 * Hk, D, dtype=dtype).split((Hk, Hk), 1)
        off_q, off_k = offsets_of(lens_q, first), offsets_of(lens_k, first)
    do = randn(seed + 2, Tq, H, D, dtype=dtype)
    scale = 1.3 * D ** -0.5
    ref = attention(q, k, v, spans_of(lens_q, lens_k, first, first), causal, scale, do)
    o, lse = sdgp.sdgp_attention(q, k, v, off_q, off_k, causal=causal, scale=scale)
    check(o, ref, "o")
    check(lse, ref, "lse")
    dq, dk, dv = sdgp.sdgp_attention_bwd(do, q, k, v, o, lse, off_q, off_k, causal=causal, scale=scale)
    check(dq, ref, "dq")
    check(dk, ref, "dk")
    check(dv, ref, "dv")
    return o, lse, dq, dk, dv


LENGTHS = [[1], [2, 1, 3], [31, 32, 33], [63, 64, 65, 1], [127, 128, 129], [0, 5, 0, 0, 70, 0], [300, 1, 17]]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", LENGTHS)
@pytest.mark.parametrize("heads", [(1, 1, 64), (4, 2, 128), (6, 2, 96)])
def test_packed(lens, heads, causal, dtype):
    packed(lens, lens, dtype, *heads, causal)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [1, 7, 8, 33, 40, 63, 65, 80, 97, 100, 127])
def test_head_sizes(D, dtype):
    packed([70, 5], [70, 5], dtype, 3, 1, D, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", [([3, 40, 1], [50, 40, 130]), ([40, 3, 7], [3, 0, 9]), ([200], [7]), ([0, 4], [6, 0]), ([1, 1, 1], [1, 700, 33])])
def test_queries_and_keys_of_different_lengths(lens, causal, dtype):
    """Also queries in front of the first key (causal), and sequences without keys: rows that see nothing."""
    packed(*lens, dtype, 4, 2, 64, causal)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tokens_without_a_sequence(dtype):
    o, lse, dq, dk, dv = packed([40, 100], [40, 100], dtype, 4, 2, 64, True, first=9, behind=150)
    for t in (o, dq, dk, dv):
        assert not t[:9].any() and not t[149:].any()
    assert bool((lse[:9] == -math.inf).all()) and bool((lse[149:] == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", [([100], [4000]), ([60, 41, 5], [2500, 1, 1000])])
def test_keys_in_parts(lens, dtype):
    """Few workgroups of many rows: the keys are cut into parts that are joined."""
    assert sdgp.binding._need("sdgp_attention_workspace", len(lens[0]), sum(lens[0]), sum(lens[1]), 4, 4, 64, 1) > 0
    packed(*lens, dtype, 4, 4, 64, True)
    packed(*lens, dtype, 2, 1, 128, False)


def test_many_sequences():
    """More than a wavefront's lanes look at at once."""
    lens = [(7 * i) % 13 for i in range(200)]
    packed(lens, lens, BF16, 2, 1, 64, True)


@pytest.mark.parametrize("first, behind", [(0, 0), (7, 300)])
def test_thousands_of_sequences(first, behind):
    """As batches of the sequences of each length: one block of keys and rows each, so the same sums, to the bit."""
    lens = [(7 * i) % 5 for i in range(9000)]
    T, (H, Hk, D) = first + sum(lens) + behind, (4, 2, 64)
    q, k, v, do = (randn(i, T, h, D, dtype=BF16) for i, h in enumerate((H, Hk, Hk, H)))
    offsets = offsets_of(lens, first)
    o, lse = sdgp.sdgp_attention(q, k, v, offsets)
    out = (o, lse, *sdgp.sdgp_attention_bwd(do, q, k, v, o, lse, offsets))
    starts, n_of = offsets[:-1].long(), torch.tensor(lens, device="cuda")
    for n in range(1, 5):
        at = starts[n_of == n][:, None] + torch.arange(n, device="cuda")
        batch = [t[at] for t in (q, k, v, do)]
        bo, blse = sdgp.sdgp_attention(*batch[:3])
        for got, want in zip(out, (bo, blse, *sdgp.sdgp_attention_bwd(batch[3], *batch[:3], bo, blse))):
            assert torch.equal(got[at], want)
    for t in (o, *out[2:]):
        assert not t[:first].any() and not t[T - behind:].any()
    assert bool((lse[:first] == -math.inf).all()) and bool((lse[T - behind:] == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 1, 128), (5, 1, 80), (40, 1, 32)])
@pytest.mark.parametrize("tokens", [1, 3])
def test_cache(tokens, heads, dtype):
    """The last tokens of sequences that fill their cache unevenly; what lies behind their lengths is not looked at."""
    H, Hk, D = heads
    lengths, L = [0, 1, 2, 31, 32, 33, 127, 128, 129, 500, 900, 1000], 1000
    B = len(lengths)
    q, k, v = randn(1, B, tokens, H, D, dtype=dtype), randn(2, B, L, Hk, D, dtype=dtype), randn(3, B, L, Hk, D, dtype=dtype)
    spans = [(i * tokens, (i + 1) * tokens, i * L, i * L + n) for i, n in enumerate(lengths)]
    ref = attention(q.view(-1, H, D), k.view(-1, Hk, D), v.view(-1, Hk, D), spans, True, D ** -0.5)
    for i, n in enumerate(lengths):
        k[i, n:], v[i, n:] = math.nan, math.inf
    o, lse = sdgp.sdgp_attention(q, k, v, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    check(o.view(-1, H, D), ref, "o")
    check(lse.view(-1, H), ref, "lse")


def test_a_batch_is_packed_sequences_of_one_length():
    q, k, v, do = (randn(i, 3, 50, h, 64, dtype=BF16) for i, h in enumerate((4, 2, 2, 4)))
    off = offsets_of([50] * 3)
    flat = [t.view(150, -1, 64) for t in (q, k, v, do)]
    o, lse = sdgp.sdgp_attention(q, k, v)
    o2, lse2 = sdgp.sdgp_attention(*flat[:3], off)
    assert torch.equal(o.view_as(o2), o2) and torch.equal(lse.view_as(lse2), lse2)
    for a, b in zip(sdgp.sdgp_attention_bwd(do, q, k, v, o, lse), sdgp.sdgp_attention_bwd(flat[3], *flat[:3], o2, lse2, off)):
        assert torch.equal(a.view_as(b), b)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_alignment(dtype):
    """Heads in front of tokens, heads that share memory, rows that begin anywhere."""
    T, H, Hk, D = 70, 4, 2, 40
    base = randn(0, H, T, D + 3, dtype=dtype)
    q = base[:, :, 1:D + 1].transpose(0, 1)
    k = randn(1, 1 + T * D, dtype=dtype)[1:].view(T, 1, D).expand(T, Hk, D)
    v = randn(2, T, D, Hk, dtype=dtype).transpose(1, 2).contiguous()
    off = offsets_of([30, 40])
    got = sdgp.sdgp_attention(q, k, v, off)
    want = sdgp.sdgp_attention(q.contiguous(), k.contiguous(), v, off)
    assert all(map(torch.equal, got, want))
    do = randn(3, T, H, D, dtype=dtype)
    for a, b in zip(sdgp.sdgp_attention_bwd(do, q, k, v, *got, off), sdgp.sdgp_attention_bwd(do, q.contiguous(), k.contiguous(), v, *got, off)):
        assert torch.equal(a, b)
    with pytest.raises(ValueError, match="stride 1"):
        sdgp.sdgp_attention(randn(2, T, D, H, dtype=dtype).transpose(1, 2), k, v, off)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_far_scores(dtype):
    """Scores of some hundreds, one key that is nearly all of the softmax, and rows of equal keys."""
    q, k, v = (randn(i, 130, 2, 64, dtype=dtype) for i in range(3))
    k[40:80] = k[40:41]
    do, off = randn(3, 130, 2, 64, dtype=dtype), offsets_of([130])
    for scale in (6.0, 1e-6):
        ref = attention(q, k, v, [(0, 130, 0, 130)], True, scale, do)
        o, lse = sdgp.sdgp_attention(q, k, v, off, scale=scale)
        check(o, ref, "o")
        check(lse, ref, "lse")
        for name, t in zip(("dq", "dk", "dv"), sdgp.sdgp_attention_bwd(do, q, k, v, o, lse, off, scale=scale)):
            check(t, ref, name)


def test_nan_stays_in_its_sequence_and_heads():
    q, k, v, do = (randn(i, 150, h, 64, dtype=BF16) for i, h in enumerate((4, 2, 2, 4)))
    off = offsets_of([50, 50, 50])
    clean = sdgp.sdgp_attention(q, k, v, off)
    clean_grads = sdgp.sdgp_attention_bwd(do, q, k, v, *clean, off)
    for t in (k, v):
        t[60, 1] = math.nan
    got = sdgp.sdgp_attention(q, k, v, off)
    grads = sdgp.sdgp_attention_bwd(do, q, k, v, *got, off)
    for a, b in zip((*got, *grads), (*clean, *clean_grads)):
        heads = a.shape[1] // 2                                             # of the first key head
        assert torch.equal(a[:, :heads], b[:, :heads]) and torch.equal(a[:50], b[:50]) and torch.equal(a[100:], b[100:])
    assert bool(got[0][60:100, 2:].isnan().all())


def test_same_bits_from_call_to_call():
    q, k, v, do = (randn(i, 500, h, 128, dtype=BF16) for i, h in enumerate((8, 2, 2, 8)))
    off = offsets_of([200, 300])
    a = sdgp.sdgp_attention(q, k, v, off)
    g = sdgp.sdgp_attention_bwd(do, q, k, v, *a, off)
    for _ in range(3):
        b = sdgp.sdgp_attention(q, k, v, off)
        assert all(map(torch.equal, a, b)) and all(map(torch.equal, g, sdgp.sdgp_attention_bwd(do, q, k, v, *b, off)))


@pytest.mark.parametrize("bad", [[0, 90, 50, 100], [-5, 30, 60, 100], [0, 50, 1000, 2000000000], [100, 50, 20, 0]])
def test_wrong_offsets_touch_nothing_outside(bad):
    """Results are anyone's guess, but memory around the tensors stays as it was."""
    T, H, D = 100, 2, 64
    q, k, v, do = (randn(i, T, H, D, dtype=BF16) for i in range(4))
    off = torch.tensor(bad, dtype=torch.int32, device="cuda")
    o, lse = sdgp.sdgp_attention(q, k, v, off)
    sdgp.sdgp_attention_bwd(do, q, k, v, o, lse, off)
    torch.cuda.synchronize()
    good = offsets_of([30, 30, 40])
    ref = attention(q, k, v, spans_of([30, 30, 40], [30, 30, 40]), True, D ** -0.5)
    check(sdgp.sdgp_attention(q, k, v, good)[0], ref, "o")


def test_offsets_that_pass_32_bits():
    """A cache of more than 2^31 values (and 2^32 bytes): all keys score 0 but the last ones of the second sequence."""
    L, Hk, D = (1 << 20) + 5, 8, 128
    k, v = (torch.zeros(2, L, Hk, D, dtype=BF16, device="cuda") for _ in range(2))
    q = randn(0, 2, 1, 16, D, dtype=BF16)
    k[1, -1] = q[1, 0, ::2]
    v[1, -1] = randn(1, Hk, D, dtype=BF16)
    lengths = torch.tensor([L, L], dtype=torch.int32, device="cuda")
    o, lse = sdgp.sdgp_attention(q, k, v, lengths=lengths, scale=1.0)
    s = (q[1, 0].double() * k[1, -1].double().repeat_interleave(2, 0)).sum(1)
    want = torch.logaddexp(s, torch.full_like(s, math.log(L - 1)))
    assert float((lse[1, 0].double() - want).abs().max()) <= 2.0 ** -10 and float((lse[0, 0].double() - math.log(L)).abs().max()) <= 2.0 ** -10
    p = torch.exp(s - want)[:, None]
    value = p * v[1, -1].double().repeat_interleave(2, 0)
    # p is rounded by 2^-8, and off by 2^-16 for a score of some hundred in 24 bits; storing rounds by 2^-8
    assert bool(((o[1, 0].double() - value).abs() <= (2 * 2.0 ** -8 + 2.0 ** -15) * value.abs() + 1e-30).all()) and not o[0].any()
    del k, v, o


def test_gradients_whose_offsets_pass_32_bits():
    """2^31 values of queries: 65536 short sequences, the last ones against 64 bits."""
    B, L, H, D = 1 << 16, 16, 16, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, do = (torch.randn(B, L, H, D, dtype=BF16, device="cuda", generator=g) for _ in range(4))
    o, lse = sdgp.sdgp_attention(q, k, v)
    grads = sdgp.sdgp_attention_bwd(do, q, k, v, o, lse)
    flat = [t[-3:].reshape(3 * L, H, D) for t in (q, k, v, do)]
    ref = attention(*flat[:3], spans_of([L] * 3, [L] * 3), True, D ** -0.5, flat[3])
    check(o[-3:].reshape(3 * L, H, D), ref, "o")
    for name, t in zip(("dq", "dk", "dv"), grads):
        check(t[-3:].reshape(3 * L, H, D), ref, name)

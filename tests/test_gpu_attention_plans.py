"""Attention and its gradients against 64 bits in the plans that only larger calls take: tiles in the order of their work, row
tiles of four wavefronts over several tiles of keys, keys' gradients from parts, groups wider than a tile."""
import pytest
import torch

import paper_2202_00774_amd as sdgp
from attention_reference import attention, check, spans_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def randn(seed, *shape, dtype=F32):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def offsets_of(lens, first):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def around(lens_q, lens_k, dtype, H, Hk, D, causal, first=0, behind=0):
    """Forward and backward, with tokens in front of the first sequence and behind the last."""
    Tq, Tk = first + sum(lens_q) + behind, first + sum(lens_k) + behind
    q, k, v, do = (randn(i, T, h, D, dtype=dtype) for i, (T, h) in enumerate(((Tq, H), (Tk, Hk), (Tk, Hk), (Tq, H))))
    off_q, off_k, scale = offsets_of(lens_q, first), offsets_of(lens_k, first), D ** -0.5
    ref = attention(q, k, v, spans_of(lens_q, lens_k, first, first), causal, scale, do)
    o, lse = sdgp.sdgp_attention(q, k, v, off_q, off_k, causal=causal)
    check(o, ref, "o")
    check(lse, ref, "lse")
    for name, t in zip(("dq", "dk", "dv"), sdgp.sdgp_attention_bwd(do, q, k, v, o, lse, off_q, off_k, causal=causal)):
        check(t, ref, name)


def ceil(a, b):
    return (a + b - 1) // b


# More than 512 workgroups, 2 to 62 sequences, 512 tokens a sequence and more: forward tiles of 128 rows, gradients of the keys in tiles of
# 128 (bf16) or 64 (fp32), each key head's.
ORDERED = [([1500, 40, 700], [1500, 40, 700]), ([1100, 1, 0, 1099], [700, 300, 64, 1500]), ([513, 2047], [2047, 513])]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", ORDERED)
@pytest.mark.parametrize("first, behind", [(0, 0), (5, 200)])
def test_tiles_in_the_order_of_their_work(lens, first, behind, causal, dtype):
    (lens_q, lens_k), S, H, Hk = lens, len(lens[0]), 64, 32
    Tq, Tk = first + sum(lens_q) + behind, first + sum(lens_k) + behind
    assert 2 <= S <= 62 and Tq >= 512 * S
    assert (Tq * (H // Hk) // 128 + S + 2) * Hk > 512 and (Tk // (128 if dtype == BF16 else 64) + S + 2) * Hk > 512
    around(lens_q, lens_k, dtype, H, Hk, 24, causal, first, behind)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_as_many_sequences_as_are_ordered(dtype):
    """62, which with the tokens in front and behind fill a wavefront's lanes; most of the work in the last ones."""
    lens = [(i * i * 37) % 97 for i in range(54)] + [6000, 1, 3700, 129, 9000, 511, 9000, 2100]
    assert len(lens) == 62 and sum(lens) >= 512 * 62
    around(lens, lens, dtype, 4, 2, 16, True, 3, 50)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [128, 80, 64, 33])
def test_rows_of_four_wavefronts_over_several_tiles_of_keys(D, causal, dtype):
    """512 workgroups of 128 rows and more, each of which passes over three to seven tiles of keys."""
    lens = [200, 190, 201, 161] * 22
    H, Hk = 6, 3
    assert len(lens) * ceil(sum(lens) // len(lens) * (H // Hk), 128) * Hk >= 512
    around(lens, lens, dtype, H, Hk, D, causal)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("tokens, G, D", [(1099, 4, 33), (1024, 1, 64), (700, 3, 96), (1500, 2, 128), (513, 1, 7)])
def test_gradients_of_keys_from_parts(tokens, G, D, causal, dtype):
    """Sums of two to sixteen parts that a second kernel adds up, four values at once and the last ones of odd counts singly."""
    size = sdgp.binding._need("sdgp_attention_bwd_workspace", 1, tokens, tokens, G, 1, D, 1 if dtype == BF16 else 0)
    parts = (size // 4 - 2 * ceil(tokens * G, 4) * 4) // (2 * tokens * D)
    assert 2 <= parts <= 16
    around([tokens], [tokens], dtype, G, 1, D, causal)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("G", [33, 40, 65, 130])
@pytest.mark.parametrize("D", [128, 64, 20])
def test_groups_wider_than_a_tile(G, D, causal, dtype):
    """More query heads to a key head than a tile of the keys' gradients has rows (32 or 64)."""
    around([70, 0, 5], [60, 3, 40], dtype, 2 * G, 2, D, causal, 1, 2)
    around([130], [130], dtype, G, 1, D, causal)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T, first", [(1, 0), (300, 0), (300, 70)])
def test_no_sequences(T, first, dtype):
    """Offsets of one entry: no token belongs to a sequence."""
    q, k, v, do = (randn(i, T, h, 64, dtype=dtype) for i, h in enumerate((4, 2, 2, 4)))
    offsets = torch.tensor([first], dtype=torch.int32, device="cuda")
    o, lse = sdgp.sdgp_attention(q, k, v, offsets)
    assert not o.any() and bool((lse == -float("inf")).all())
    for t in sdgp.sdgp_attention_bwd(do, q, k, v, o, lse, offsets):
        assert not t.any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_same_bits_from_call_to_call(dtype):
    lens = [1500, 40, 700]
    q, k, v, do = (randn(i, sum(lens), h, 24, dtype=dtype) for i, h in enumerate((64, 32, 32, 64)))
    offsets = offsets_of(lens, 0)
    a = sdgp.sdgp_attention(q, k, v, offsets)
    g = sdgp.sdgp_attention_bwd(do, q, k, v, *a, offsets)
    for _ in range(3):
        b = sdgp.sdgp_attention(q, k, v, offsets)
        assert all(map(torch.equal, a, b)) and all(map(torch.equal, g, sdgp.sdgp_attention_bwd(do, q, k, v, *b, offsets)))

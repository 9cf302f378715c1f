"""Token log probabilities, entropy, top alternatives and their gradient against their definition in 64 bits.

Bounds, with e = 2^-24 (one fp32 rounding) and z = scale (x - max):
  * a term 2^(c (x - max)) of the sums carries at most 3 roundings of an exponent of z, so 3 e |z| relative, and the
    2 e of the exponential itself; |z| e^z <= 0.37, so over the sum that is at most 5 e (the largest term is 1).  A sum
    of n terms in any order adds n e.  Chains are at most V / 64 + 32 long (64 lanes at least share a row).
  * so ln s is off by at most N e, N = V / 64 + 40;  logp adds three roundings of z and ln s;  the entropy adds
    the same relative error of sum p |z| twice (numerator, quotient);
  * p carries the error of its logarithm, (N + 4 |z|) e; every gradient term that many e of its own size, and the
    result one rounding to its type (2^-8 in bf16).  Probabilities below 2^-126 may count as 0: their term is that times
    scale (|g| + |h| |ln p|) with |ln p| + entropy below 110 where they are not 0 anyway; V of them may be missing from the
    entropy, which every term of its gradient holds.
"""
import numpy as np
import pytest
import torch

import paper_2202_00774_amd as sdgp

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
DT = [torch.float32, torch.bfloat16]


def reference(x, tokens, scale, top, g=None, h=None):
    """x [rows, V] float64, in numpy; a row at a time."""
    rows, V = x.shape
    out = {"logp": np.zeros(rows), "entropy": np.zeros(rows), "ids": np.full((rows, top), -1, np.int64), "top": np.full((rows, top), -np.inf),
           "lnp": np.full((rows, V), -np.inf), "z": np.zeros((rows, V)), "d": np.zeros((rows, V)), "size": np.zeros((rows, V))}
    for r in range(rows):
        if np.isnan(x[r]).any() or (x[r] == np.inf).any():
            for k in ("logp", "entropy", "top", "lnp", "d"):
                out[k][r] = np.nan
            if tokens[r] < 0:
                out["logp"][r] = 0.0
            continue
        m = x[r].max()
        if m > -np.inf:
            z = scale * (x[r] - m)
            lnp = z - np.log(np.exp(z).sum())
            p = np.exp(lnp)
            out["entropy"][r] = -(p * np.where(p > 0, lnp, 0)).sum()
            order = np.lexsort((np.arange(V), -x[r]))[:top]
            order = order[x[r][order] > -np.inf]
            out["ids"][r, :len(order)], out["top"][r, :len(order)] = order, lnp[order]
            out["lnp"][r], out["z"][r] = lnp, np.maximum(z, -1e6)
            if g is not None:
                gr = g[r] if tokens[r] >= 0 else 0.0
                l = np.where(p > 0, lnp, 0)
                out["d"][r] = -p * (gr + h[r] * (l + out["entropy"][r]))
                out["size"][r] = p * (abs(gr) + abs(h[r]) * (abs(l) + out["entropy"][r]))
                if 0 <= tokens[r] < V:
                    out["d"][r, tokens[r]] += gr
                    out["size"][r, tokens[r]] += abs(gr)
        if tokens[r] >= 0:
            out["logp"][r] = out["lnp"][r, tokens[r]] if tokens[r] < V else np.nan
        if tokens[r] >= V and g is not None:
            out["d"][r] = np.nan
    out["d"] *= scale
    out["size"] *= scale
    return out


def near(got, want, bound, what):
    got = np.asarray(got, np.float64)
    assert got.shape == want.shape, what
    want = np.where(np.abs(want) > np.finfo(np.float32).max, np.copysign(np.inf, want), want)     # no fp32 value
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
    off = np.abs(got - want)[fine] - np.broadcast_to(bound, want.shape)[fine]
    assert (off <= 0).all(), (what, off.max(), np.abs(want[fine]).max())


def check(logits, tokens, top, scale=1.0, seed=0, token_dtype=torch.int64):
    """logits: a GPU tensor [rows, V], any row stride."""
    rows, V = logits.shape
    rng = np.random.default_rng(seed)
    x = logits.double().cpu().numpy()
    tok = torch.from_numpy(np.asarray(tokens)).to(token_dtype).cuda()
    g, h = rng.normal(size=rows).astype(np.float32), rng.normal(size=rows).astype(np.float32)
    want = reference(x, np.asarray(tokens), float(np.float32(scale)), top, g.astype(np.float64), h.astype(np.float64))
    before = logits.clone()
    logp, entropy, top_logp, top_ids, stats = sdgp.sdgp_token_logprobs(logits, tok, top=top, scale=scale)
    N = V / 64 + 40
    with np.errstate(invalid="ignore"):
        zt = np.abs(want["logp"]) + np.log(V)
        near(logp.cpu(), want["logp"], E * (N + 4 * zt), "logp")
        near(entropy.cpu(), want["entropy"], E * 3 * (N + 4) * (1 + want["entropy"]), "entropy")
        if top:
            assert np.array_equal(top_ids.cpu().numpy(), want["ids"])
            near(top_logp.cpu(), want["top"], E * (N + 4 * (np.abs(want["top"]) + np.log(V))), "top_logp")
        else:
            assert top_logp is None and top_ids is None
        d = sdgp.sdgp_token_logprobs_bwd(logits, tok, stats, entropy, torch.from_numpy(g).cuda(), torch.from_numpy(h).cuda(), scale=scale)
        assert d.dtype == logits.dtype and d.is_contiguous()
        store = 2.0 ** -8 if logits.dtype == torch.bfloat16 else E
        tiny = 2.0 ** -126 * V * (1 + scale * (np.abs(g) + 110 * np.abs(h)))[:, None]
        bound = E * (4 * N + 4 * np.abs(want["z"])) * want["size"] + store * np.abs(want["d"]) + tiny
        near(d.double().cpu(), want["d"], bound, "dlogits")
        # each gradient alone
        d = sdgp.sdgp_token_logprobs_bwd(logits, tok, stats, None, torch.from_numpy(g).cuda(), None, scale=scale)
        alone = reference(x, np.asarray(tokens), float(np.float32(scale)), 0, g.astype(np.float64), 0 * h)
        near(d.double().cpu(), alone["d"], E * (4 * N + 4 * np.abs(alone["z"])) * alone["size"] + store * np.abs(alone["d"]) + tiny, "from logp")
        d = sdgp.sdgp_token_logprobs_bwd(logits, None, stats, entropy, None, torch.from_numpy(h).cuda(), scale=scale)
        none = np.full(rows, -1)
        alone = reference(x, none, float(np.float32(scale)), 0, 0.0 * g, h.astype(np.float64))
        near(d.double().cpu(), alone["d"], E * (4 * N + 4 * np.abs(alone["z"])) * alone["size"] + store * np.abs(alone["d"]) + tiny, "from entropy")
    as_int = torch.int16 if logits.dtype == torch.bfloat16 else torch.int32
    assert torch.equal(logits.contiguous().view(as_int), before.contiguous().view(as_int))
    # the same bits from call to call
    again = sdgp.sdgp_token_logprobs(logits, tok, top=top, scale=scale)
    for a, b in zip((logp, entropy, top_logp, stats), (again[0], again[1], again[2], again[4])):
        assert a is None or torch.equal(a.view(torch.int32), b.view(torch.int32))
    return logp, entropy, top_logp, top_ids, stats


def random_logits(rows, V, dtype, seed, spread=3.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(rows, V, device="cuda", generator=g) * spread).to(dtype)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 64, 65, 255, 256, 257, 511, 1000, 2047, 2049, 4099, 8193, 16385, 50021])
def test_widths(V, dtype):
    for rows in (1, 3, 6):
        x = random_logits(rows, V, dtype, 100 * V + rows)
        tokens = np.random.default_rng(V).integers(-1, V, rows)
        check(x, tokens, min(V, 5), scale=0.7, seed=V)
        check(x, tokens, 0, seed=V, token_dtype=torch.int32)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("top", [1, 2, 31, 63, 64])
def test_number_of_alternatives(top, dtype):
    for V in (64, 300, 5000):
        check(random_logits(4, V, dtype, top + V), [0, V - 1, -100, V // 2], top)


@pytest.mark.parametrize("dtype", DT)
def test_rows_that_start_anywhere_and_lie_apart(dtype):
    """A vocabulary cut out of wider rows: every offset within 16 bytes, odd strides."""
    for off in range(9):
        for pad in (0, 1, 3):
            wide = random_logits(5, 1003 + off + pad, dtype, off)
            check(wide[:, off:off + 1003], [0, 1002, 17, -1, 500], 4, seed=off)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows", [255, 256, 700, 1025, 2100])
def test_many_rows(rows, dtype):
    for V in (5, 130, 1000):
        check(random_logits(rows, V, dtype, rows), np.random.default_rng(rows).integers(-1, V, rows), min(V, 3))


@pytest.mark.parametrize("dtype", DT)
def test_few_long_rows(dtype):
    for rows, V in ((1, 131072), (2, 131071), (4, 100003), (1, 300007)):
        check(random_logits(rows, V, dtype, V), [V - 1] * rows, 8, scale=1.25)
        check(random_logits(rows, V, dtype, V), [0] * rows, 64)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("V", [9, 300, 20011, 140001])
def test_equal_logits_come_in_the_order_of_their_index(V, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    few = torch.randint(0, 3, (4, V), device="cuda", generator=g).to(dtype)
    few[1] = 0.0
    few[1, ::2] = -0.0                                    # equal to +0
    few[2] = few[2, 0]
    check(few, [0, 1, 2, V - 1], min(V, 64))
    check(few, [0, 1, 2, V - 1], min(V, 5))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("V", [70, 3001, 70001])
def test_ordered_rows(V, dtype):
    """Rising logits: every one is an alternative when it is met; falling: only the first are."""
    up = torch.linspace(-5, 5, V, device="cuda").to(dtype)
    check(torch.stack([up, up.flip(0), torch.zeros_like(up)]), [0, 0, 1], 10)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("V", [1, 5, 64, 1000, 4099, 70001])
def test_masks_and_rows_that_leave_nothing(V, dtype):
    lowest = torch.finfo(dtype).min
    x = random_logits(9, V, dtype, V)
    x[0] = -np.inf                                        # nothing left
    x[1] = -np.inf
    x[1, V // 2] = 3.0                                    # one token left: probability 1
    x[2] = lowest                                         # a mask of the lowest value throughout: all alike
    x[3, ::2] = lowest
    x[4, 1:] = -np.inf                                    # fewer left than alternatives
    x[5, ::3] = -np.inf
    x[6, V - 1] = np.inf
    x[7, V // 3] = np.nan
    x[8] = torch.finfo(dtype).max                         # the largest value throughout
    top = min(V, 6)
    tokens = [0, V // 2, 0, min(V - 1, 1), min(V - 1, 1), 0, 0, V - 1, V - 1]
    logp, entropy, top_logp, top_ids, _ = check(x, tokens, top, scale=1.5)
    assert logp[0] == -np.inf and entropy[0] == 0 and (top_ids[0] == -1).all()
    assert logp[1] == 0 and entropy[1] == 0 and top_ids[1, 0] == V // 2 and (top_ids[1, 1:] == -1).all()
    assert (top_ids[6:8] == -1).all() and torch.isnan(top_logp[6:8]).all()
    check(x, [-1] * 9, top)


@pytest.mark.parametrize("dtype", DT)
def test_tokens_outside_the_vocabulary(dtype):
    x = random_logits(6, 77, dtype, 1)
    logp, *_ = check(x, [-1, -100, 76, 77, 2**31 - 1, 0], 2)
    assert (logp[:2] == 0).all() and torch.isnan(logp[3:5]).all()
    check(x, [-2**40, -100, 76, 2**40, 2**33 + 5, 0], 2)


@pytest.mark.parametrize("dtype", DT)
def test_peaked_rows_and_scales(dtype):
    x = random_logits(4, 3000, dtype, 2, spread=1.0)
    x[:, 5] = torch.tensor([10.0, 40.0, 90.0, 1000.0])
    for scale in (0.01, 1.0, 3.0, 100.0):
        check(x, [5, 5, 6, 7], 3, scale=scale)


def test_without_tokens_in_three_dimensions_and_in_place():
    x = random_logits(6, 501, torch.bfloat16, 3)
    flat = sdgp.sdgp_token_logprobs(x, None, top=2)
    assert flat[0] is None
    cube = x.view(2, 3, 501)
    tokens = torch.arange(6, device="cuda").view(2, 3)
    logp, entropy, top_logp, top_ids, stats = sdgp.sdgp_token_logprobs(cube, tokens, top=2)
    assert logp.shape == entropy.shape == (2, 3) and top_ids.shape == top_logp.shape == (2, 3, 2) and stats.shape == (2, 3, 2)
    assert torch.equal(entropy.view(-1), flat[1]) and torch.equal(top_ids.view(6, 2), flat[3])
    g = torch.randn(2, 3, device="cuda")
    d = sdgp.sdgp_token_logprobs_bwd(cube, tokens, stats, None, g)
    assert d.shape == cube.shape
    own = cube.clone()
    assert sdgp.sdgp_token_logprobs_bwd(own, tokens, stats, None, g, out=own) is own
    assert torch.equal(own, d)
    wide = torch.full((6, 600), 7.0, device="cuda", dtype=torch.bfloat16)
    sdgp.sdgp_token_logprobs_bwd(x, tokens.view(6), stats.view(6, 2), None, g.view(6), out=wide[:, 33:534])
    assert torch.equal(wide[:, 33:534], d.view(6, 501)) and (wide[:, :33] == 7).all() and (wide[:, 534:] == 7).all()
    one = sdgp.sdgp_token_logprobs(x[0], torch.tensor(4, device="cuda"), top=2)
    assert one[0].shape == () and torch.equal(one[3], flat[3][0])


def test_no_rows():
    x = torch.empty(0, 9, device="cuda")
    logp, entropy, top_logp, top_ids, stats = sdgp.sdgp_token_logprobs(x, torch.empty(0, dtype=torch.int64, device="cuda"), top=3)
    assert logp.shape == (0,) and top_ids.shape == (0, 3)
    assert sdgp.sdgp_token_logprobs_bwd(x, torch.empty(0, dtype=torch.int64, device="cuda"), stats, None, logp).shape == (0, 9)


def test_gradient_against_differences():
    """A step of 1e-3 along a random direction, both sides of the logits, the function in 64 bits: the difference
    quotient is off by its third derivative, below 1e-6 of the gradients' size (the function's scale is 1)."""
    x = random_logits(3, 400, torch.float32, 4)
    tokens = np.array([1, 399, -1])
    tok = torch.from_numpy(tokens).cuda()
    g, h = torch.tensor([0.7, -1.3, 2.0], device="cuda"), torch.tensor([0.4, 0.9, -1.1], device="cuda")
    _, entropy, _, _, stats = sdgp.sdgp_token_logprobs(x, tok, scale=1.5)
    d = sdgp.sdgp_token_logprobs_bwd(x, tok, stats, entropy, g, h, scale=1.5).double().cpu().numpy()
    xs, rng, step = x.double().cpu().numpy(), np.random.default_rng(0), 1e-3

    def value(at, r):
        want = reference(at[r:r + 1], tokens[r:r + 1], 1.5, 0)
        return g[r].item() * want["logp"][0] + h[r].item() * want["entropy"][0]

    for _ in range(5):
        v = rng.normal(size=xs.shape)
        for r in range(3):
            quotient = (value(xs + step * v, r) - value(xs - step * v, r)) / (2 * step)
            assert abs(quotient - (d[r] * v[r]).sum()) <= 1e-4


def test_refusals():
    x = random_logits(4, 32, torch.float32, 5)
    tok = torch.zeros(4, dtype=torch.int64, device="cuda")
    for bad in (dict(top=33), dict(top=-1), dict(scale=0.0), dict(scale=float("nan"))):
        with pytest.raises(sdgp.SdgpError):
            sdgp.sdgp_token_logprobs(x, tok, **bad)
    with pytest.raises(TypeError):
        sdgp.sdgp_token_logprobs(x.half(), tok)
    for bad in (tok[:3], tok.float(), tok.cpu(), tok.view(2, 2)):
        with pytest.raises(ValueError):
            sdgp.sdgp_token_logprobs(x, bad)
    for bad in (x.t(), x[:, ::2], x[:1].expand(4, 32)):
        with pytest.raises(ValueError):
            sdgp.sdgp_token_logprobs(bad, None)
    with pytest.raises(sdgp.SdgpError):
        sdgp.sdgp_token_logprobs(x[:, :0], None)
    logp, entropy, _, _, stats = sdgp.sdgp_token_logprobs(x, tok)
    for args in ((x, tok, stats, entropy, None, None), (x, None, stats, None, logp, None), (x, tok, stats, None, None, logp),
                 (x, tok, stats[:3], None, logp, None), (x, tok, stats, None, logp.double(), None)):
        with pytest.raises(ValueError):
            sdgp.sdgp_token_logprobs_bwd(*args)
    with pytest.raises(ValueError):
        sdgp.sdgp_token_logprobs_bwd(x, tok, stats, None, logp, out=torch.empty(4, 31, device="cuda"))


def test_another_stream():
    x = random_logits(300, 5003, torch.bfloat16, 6)
    tok = torch.arange(300, device="cuda")
    want = sdgp.sdgp_token_logprobs(x, tok, top=4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = x.clone()
        got = sdgp.sdgp_token_logprobs(late, tok, top=4)
        d = sdgp.sdgp_token_logprobs_bwd(late, tok, got[4], None, got[0])
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[3], want[3])
    assert torch.equal(d, sdgp.sdgp_token_logprobs_bwd(x, tok, want[4], None, want[0]))


@pytest.mark.parametrize("dtype,V", [(torch.bfloat16, 65536), (torch.bfloat16, 65537), (torch.float32, 33000)])
def test_logits_larger_than_the_caches(dtype, V):
    """Above 256 MB logits are read, above 80 MB gradients written, past the caches.  Rows are problems of their own: parts of
    525 of them (69 MB), cut the same way, give the same bits."""
    x = random_logits(2100, V, dtype, V)
    x[7, ::3] = -np.inf
    assert x.numel() * x.element_size() > 256 << 20
    tokens = torch.randint(-1, V, (2100,), device="cuda")
    g = torch.randn(2100, device="cuda")
    whole = sdgp.sdgp_token_logprobs(x, tokens, top=2)
    d = sdgp.sdgp_token_logprobs_bwd(x, tokens, whole[4], whole[1], g, g)
    for lo in range(0, 2100, 525):
        cut = slice(lo, lo + 525)
        part = sdgp.sdgp_token_logprobs(x[cut], tokens[cut], top=2)
        for a, b in zip(whole, part):
            assert torch.equal(a[cut], b)
        assert torch.equal(d[cut], sdgp.sdgp_token_logprobs_bwd(x[cut], tokens[cut], part[4], part[1], g[cut], g[cut]))


def test_rows_further_apart_than_32_bits_count():
    room = torch.empty(2**32 + 40000, dtype=torch.bfloat16, device="cuda")
    x = room.as_strided((3, 9001), (2**31 + 5, 1))
    near_by = random_logits(3, 9001, torch.bfloat16, 77)
    x.copy_(near_by)
    tokens, g = torch.tensor([9000, 0, 5], device="cuda"), torch.randn(3, device="cuda")
    far, want = sdgp.sdgp_token_logprobs(x, tokens, top=4), sdgp.sdgp_token_logprobs(near_by, tokens, top=4)
    for a, b in zip(far, want):
        assert torch.equal(a, b)
    sdgp.sdgp_token_logprobs_bwd(x, tokens, far[4], far[1], g, g, out=x)
    assert torch.equal(x, sdgp.sdgp_token_logprobs_bwd(near_by, tokens, want[4], want[1], g, g))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("top", [1, 3, 4, 5, 8, 9, 16, 17, 32, 33, 64])
def test_alternatives_of_which_the_first_chunk_has_all_few_or_none(top, dtype):
    """A row's first 4096 bf16 or 2048 fp32 logits give a bound for the rest.  600 rows: none is cut into pieces."""
    chunk, V = (4096, 9001) if dtype == torch.bfloat16 else (2048, 5001)
    g = torch.Generator()
    g.manual_seed(top)
    x = torch.randn(600, V, generator=g)
    x[1::6, :chunk] -= 20                                     # all of the best behind the first chunk
    x[2::6, chunk:] -= 20                                     # all in it
    x[3::6, :chunk] = -float("inf")                           # nothing in it
    x[4::6, : chunk - 3] = -float("inf")                      # three logits in it
    x[5::6] = torch.randint(0, 3, (100, V), generator=g).float()   # equal ones throughout
    x[0, :chunk] = 7.0
    x[6, 3:] = -float("inf")                                  # fewer than are asked for
    x = x.to(dtype)
    _, _, lp, ids, _ = sdgp.sdgp_token_logprobs(x.cuda(), None, top=top)
    x64 = x.double().numpy()
    want = np.argsort(-x64, axis=1, kind="stable")[:, :top]
    none = np.take_along_axis(x64, want, 1) == -np.inf
    assert np.array_equal(ids.cpu().numpy(), np.where(none, -1, want))
    assert np.array_equal(np.isneginf(lp.cpu().numpy()), none)

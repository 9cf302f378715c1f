"""Block norms (norm after, gate, scaled residual, norm before the next block) and their gradient against the formulas in
64 bits.

Bounds, with e = 2^-24: a sum of D terms in any order is off by at most D e of the sum of sizes; here threads share a
row, so chains are at most D / 64 + 16 long.  So a norm's factor is off by (D / 64 + 24) e relative at most (N e below),
a product of k factors adds k e, and storing adds one rounding (2^-8 bf16, e fp32).  y is compared with the formula; h
and the gradients with the formula from y as the call stored it, since that is what they are defined on.  Gradients: N e
of the size of every term that is added up, the mean's terms included.  Sums over rows: (rows + N) e of the sum of sizes.
"""
import numpy as np
import pytest
import torch

import paper_2202_00774_amd as sdgp

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
DT = [torch.float32, torch.bfloat16]


def f64(t):
    return t.detach().double().cpu().numpy()


def near(got, want, bound, what):
    got = f64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = np.abs(got - want) - bound
    assert (off <= 0).all(), (what, float(off.max()), float(np.abs(want).max()))


def make(rows, D, dtype, gate, seed, block=True, wdtype=torch.float32, weights=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    t = {"x": (2 * rnd(rows, D)).to(dtype), "u": None, "gate": None, "w_post": None, "w_pre": None}
    if weights:
        t["w_pre"] = (1 + 0.3 * rnd(D)).to(wdtype)
    if block:
        t["u"] = (0.5 * rnd(rows, D)).to(dtype)
        if weights:
            t["w_post"] = (1 + 0.3 * rnd(D)).to(wdtype)
        if gate:
            t["gate"] = rnd(gate, D).to(dtype)
    t["dy"], t["dh"] = rnd(rows, D).to(dtype), rnd(rows, D).to(dtype)
    return t


def check(t, residual_scale=1.0, eps=1e-6, pre=True, with_dy=True):
    x = t["x"]
    rows, D = x.shape
    store = 2.0 ** -8 if x.dtype == torch.bfloat16 else E
    N = D / 64 + 32
    before = {k: v.clone() for k, v in t.items() if v is not None}
    w_pre = t["w_pre"] if pre else None
    y, h, stats = sdgp.sdgp_block_norm(x, t["u"], t["gate"], t["w_post"], w_pre, residual_scale=residual_scale, eps=eps, pre=pre)
    rs = float(np.float32(residual_scale))
    one = np.ones(D)
    wp = f64(t["w_post"]) if t["w_post"] is not None else one
    wr = f64(w_pre) if w_pre is not None else one
    per = 1
    if t["u"] is None:
        assert y is x
    else:
        u = f64(t["u"])
        ru = 1 / np.sqrt((u * u).mean(1, keepdims=True) + eps)
        a = u * ru
        G = t["gate"].numel() // D if t["gate"] is not None else 0
        k = np.repeat(f64(t["gate"]).reshape(G, D), rows // G, 0) if G else np.ones((1, D))
        part = k * a * wp
        want = rs * f64(x) + part
        near(y, want, E * N * (np.abs(rs * f64(x)) + np.abs(part)) + store * np.abs(want) + 1e-38, "y")
    ys = f64(y)
    ry = 1 / np.sqrt((ys * ys).mean(1, keepdims=True) + eps)
    n = ys * ry
    if not pre:
        assert h is None
    else:
        near(h, n * wr, (E * N + store) * np.abs(n * wr) + 1e-38, "h")

    dy = t["dy"] if with_dy else None
    dh = t["dh"] if pre else None
    got = sdgp.sdgp_block_norm_bwd(dy, dh, y, stats, t["u"], t["gate"], t["w_post"], w_pre, residual_scale=residual_scale)
    dx, du, dgate, dw_post, dw_pre = got
    dY = f64(dy) if with_dy else np.zeros((rows, D))
    size = np.abs(dY)
    if pre:
        q = f64(dh) * wr
        dY = dY + ry * (q - n * (q * n).mean(1, keepdims=True))
        size = size + ry * (np.abs(q) + np.abs(n) * np.abs(q * n).mean(1, keepdims=True))
        term = f64(dh) * n
        if w_pre is not None:
            assert dw_pre.dtype == torch.float32
            near(dw_pre, term.sum(0), E * (rows + N) * np.abs(term).sum(0) + 1e-38, "dw_pre")
    if w_pre is None:
        assert dw_pre is None
    f = rs if t["u"] is not None else 1.0
    near(dx, f * dY, abs(f) * E * 4 * N * size + store * np.abs(f * dY) + 1e-38, "dx")
    if t["u"] is None:
        assert du is None and dgate is None and dw_post is None
    else:
        q = dY * k * wp
        qs = size * np.abs(k * wp)
        want = ru * (q - a * (q * a).mean(1, keepdims=True))
        near(du, want, ru * E * 8 * N * (qs + np.abs(a) * (qs * np.abs(a)).mean(1, keepdims=True)) + store * np.abs(want) + 1e-38, "du")
        if t["w_post"] is not None:
            assert dw_post.dtype == torch.float32
            near(dw_post, (dY * k * a).sum(0), E * (rows + 8 * N) * (size * np.abs(k * a)).sum(0) + 1e-38, "dw_post")
        else:
            assert dw_post is None
        if G:
            assert dgate.dtype == x.dtype and dgate.shape == t["gate"].shape
            term, sizes = (dY * a * wp).reshape(G, -1, D).sum(1), (size * np.abs(a * wp)).reshape(G, -1, D).sum(1)
            near(dgate.view(G, D), term, E * (rows // G + 8 * N) * sizes + store * np.abs(term) + 1e-38, "dgate")
        else:
            assert dgate is None
    for key, v in before.items():
        as_int = torch.int16 if v.dtype == torch.bfloat16 else torch.int32
        assert torch.equal(t[key].view(as_int), v.view(as_int)), key
    # the same bits from call to call
    again = sdgp.sdgp_block_norm_bwd(dy, dh, y, stats, t["u"], t["gate"], t["w_post"], w_pre, residual_scale=residual_scale)
    for p, q in zip(got, again):
        assert p is None or torch.equal(p, q)


WIDTHS = [1, 2, 3, 7, 8, 9, 16, 63, 64, 65, 127, 128, 200, 255, 256, 257, 512, 520, 1000, 1001, 1024, 1536, 2048, 2056, 4095, 4096, 4104, 8192, 8200, 12289, 16384, 20000]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("D", WIDTHS)
def test_widths(D, dtype):
    check(make(12, D, dtype, 1, D))
    check(make(12, D, dtype, 4, D + 1, wdtype=dtype), residual_scale=0.5)
    check(make(5, D, dtype, 5, D + 2), residual_scale=-1.25)
    check(make(3, D, dtype, 0, D + 3, weights=False))
    check(make(7, D, dtype, 0, D + 4, block=False))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,gate", [(1, 1), (2, 1), (2, 2), (63, 7), (64, 64), (257, 1), (1000, 8), (1000, 500), (1024, 1024), (2500, 1), (5000, 50), (8192, 2), (20011, 1)])
def test_rows_and_gates(rows, gate, dtype):
    for D in (24, 130, 264):
        check(make(rows, D, dtype, gate, rows + D))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("D", [40, 264, 1001, 2048])
def test_parts_left_out(D, dtype):
    t = make(37, D, dtype, 1, D)
    check(t, pre=False)                                    # no norm follows
    check(t, with_dy=False)                                # nothing comes back along the residual
    check(make(37, D, dtype, 37, D), pre=False)
    check(make(37, D, dtype, 0, D, weights=False), pre=False)
    check(make(37, D, dtype, 0, D, block=False, weights=False), with_dy=False)
    check(make(37, D, dtype, 0, D, block=False))


@pytest.mark.parametrize("dtype", DT)
def test_rows_of_zeros_and_of_very_different_sizes(dtype):
    t = make(9, 520, dtype, 1, 3)
    t["u"][0] = 0                                          # the factor is 1 / sqrt(eps)
    t["x"][1] = 0
    t["u"][1] = 0
    t["u"][2] *= 1e-4
    t["u"][3] *= 1e4
    t["x"][4] *= 1e4
    t["gate"][:, ::2] = 0                                  # gates start at zero
    check(t, eps=1e-5)


@pytest.mark.parametrize("dtype", DT)
def test_a_row_that_is_not_finite_stays_alone(dtype):
    t = make(8, 264, dtype, 8, 4)
    want_y, want_h, _ = sdgp.sdgp_block_norm(t["x"], t["u"], t["gate"], t["w_post"], t["w_pre"])
    t["u"][3, 5] = float("nan")
    t["x"][6, 7] = float("inf")
    y, h, stats = sdgp.sdgp_block_norm(t["x"], t["u"], t["gate"], t["w_post"], t["w_pre"])
    fine = [0, 1, 2, 4, 5, 7]
    assert torch.equal(y[fine], want_y[fine]) and torch.equal(h[fine], want_h[fine])
    assert torch.isnan(y[3]).all() and torch.isnan(h[3]).all() and torch.isinf(y[6, 7]) and torch.isnan(h[6, 7])
    dx, du, dgate, dw_post, dw_pre = sdgp.sdgp_block_norm_bwd(t["dy"], t["dh"], y, stats, t["u"], t["gate"], t["w_post"], t["w_pre"])
    assert torch.isfinite(dx[fine]).all() and torch.isfinite(du[fine]).all() and torch.isfinite(dgate[fine]).all()
    assert torch.isnan(dx[3]).all() and torch.isnan(dw_pre).all()


def test_tensors_that_start_anywhere():
    """Contiguous, but not on 16 bytes."""
    for dtype in DT:
        for off in (1, 2, 3, 4):
            t = make(6, 264, dtype, 2, off)
            for k, v in t.items():
                if v is not None:
                    room = torch.empty(v.numel() + 8, dtype=v.dtype, device="cuda")
                    room[off:off + v.numel()] = v.reshape(-1)
                    t[k] = room[off:off + v.numel()].view(v.shape)
            check(t)


def test_three_dimensions_and_no_rows():
    t = make(24, 96, torch.bfloat16, 4, 9)
    y, h, stats = sdgp.sdgp_block_norm(t["x"], t["u"], t["gate"], t["w_post"], t["w_pre"])
    cube = [t[k].view(4, 6, 96) for k in ("x", "u")]
    y3, h3, s3 = sdgp.sdgp_block_norm(*cube, t["gate"].view(4, 1, 96), t["w_post"], t["w_pre"])
    assert y3.shape == (4, 6, 96) and torch.equal(y3.view(24, 96), y) and torch.equal(h3.view(24, 96), h) and torch.equal(s3, stats)
    e = torch.empty(0, 96, device="cuda", dtype=torch.bfloat16)
    y, h, stats = sdgp.sdgp_block_norm(e, e, t["gate"][0], t["w_post"], t["w_pre"])
    assert y.shape == h.shape == (0, 96)
    dx, du, dgate, dw_post, dw_pre = sdgp.sdgp_block_norm_bwd(e, e, y, stats, e, t["gate"][0], t["w_post"], t["w_pre"])
    assert dx.shape == (0, 96) and (dgate == 0).all() and (dw_post == 0).all() and (dw_pre == 0).all()


def test_gradient_against_differences():
    """fp32, the function in 64 bits, a step of 1e-3 both ways: off by the third derivative, below 1e-5 here."""
    t = make(6, 40, torch.float32, 3, 11)
    y, h, stats = sdgp.sdgp_block_norm(t["x"], t["u"], t["gate"], t["w_post"], t["w_pre"], residual_scale=0.75)
    grads = sdgp.sdgp_block_norm_bwd(t["dy"], t["dh"], y, stats, t["u"], t["gate"], t["w_post"], t["w_pre"], residual_scale=0.75)
    names = ("x", "u", "gate", "w_post", "w_pre")
    at = {k: f64(t[k]) for k in names}

    def value(p):
        norm = lambda v: v / np.sqrt((v * v).mean(1, keepdims=True) + 1e-6)  # noqa: E731
        yy = 0.75 * p["x"] + np.repeat(p["gate"], 2, 0) * norm(p["u"]) * p["w_post"]
        return (yy * f64(t["dy"])).sum() + (norm(yy) * p["w_pre"] * f64(t["dh"])).sum()

    rng = np.random.default_rng(1)
    for name, grad in zip(names, grads):
        for _ in range(3):
            v = rng.normal(size=at[name].shape)
            q = (value({**at, name: at[name] + 1e-3 * v}) - value({**at, name: at[name] - 1e-3 * v})) / 2e-3
            dot = (f64(grad) * v).sum()
            assert abs(q - dot) <= 1e-3 * max(1.0, abs(dot)), (name, q, dot)


def test_refusals():
    t = make(6, 32, torch.bfloat16, 3, 12)
    ok = lambda **k: sdgp.sdgp_block_norm(*[{**t, **k}[n] for n in ("x", "u", "gate", "w_post", "w_pre")])  # noqa: E731
    ok()
    for bad in (dict(u=t["u"][:5]), dict(u=t["u"].float()), dict(gate=t["gate"].float()), dict(gate=t["x"][:4]), dict(gate=t["gate"][:, :16].contiguous()),
                dict(w_pre=t["w_pre"][:31]), dict(w_post=t["w_post"].to(torch.bfloat16)), dict(u=None), dict(x=t["x"].t()), dict(w_pre=t["w_pre"].cpu())):
        with pytest.raises(ValueError):
            ok(**bad)
    with pytest.raises(TypeError):
        ok(x=t["x"].half(), u=t["u"].half(), gate=t["gate"].half())
    with pytest.raises(ValueError):
        sdgp.sdgp_block_norm(t["x"], pre=False)
    with pytest.raises(sdgp.SdgpError):
        sdgp.sdgp_block_norm(t["x"], eps=-1.0)
    y, h, stats = ok()
    with pytest.raises(ValueError):
        sdgp.sdgp_block_norm_bwd(None, None, y, stats)
    with pytest.raises(ValueError):
        sdgp.sdgp_block_norm_bwd(t["dy"], None, y, stats, t["u"], w_pre=t["w_pre"])
    with pytest.raises(ValueError):
        sdgp.sdgp_block_norm_bwd(t["dy"], t["dh"], y, stats[:, :5], t["u"])


def test_another_stream():
    t = make(600, 264, torch.bfloat16, 1, 13)
    want = sdgp.sdgp_block_norm(t["x"], t["u"], t["gate"], t["w_post"], t["w_pre"])
    grads = sdgp.sdgp_block_norm_bwd(t["dy"], t["dh"], want[0], want[2], t["u"], t["gate"], t["w_post"], t["w_pre"])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = {k: v.clone() for k, v in t.items()}
        got = sdgp.sdgp_block_norm(late["x"], late["u"], late["gate"], late["w_post"], late["w_pre"])
        more = sdgp.sdgp_block_norm_bwd(late["dy"], late["dh"], got[0], got[2], late["u"], late["gate"], late["w_post"], late["w_pre"])
    side.synchronize()
    for p, q in zip((*want, *grads), (*got, *more)):
        assert torch.equal(p, q)


@pytest.mark.parametrize("dtype,rows,D,gate", [(torch.bfloat16, 36000, 2048, 1), (torch.float32, 9001, 4097, 1), (torch.bfloat16, 18000, 4096, 4)])
def test_tensors_larger_than_the_caches(dtype, rows, D, gate):
    """More than 128 MB a tensor: written and cut differently.  Every row is its own problem, so a part of the rows gives
    the same bits; the sums over rows are the parts' sums, to (rows) e of the sum of sizes each side."""
    t = make(rows, D, dtype, gate, D)
    assert rows * D * t["x"].element_size() > 128 << 20
    y, h, stats = sdgp.sdgp_block_norm(t["x"], t["u"], t["gate"], t["w_post"], t["w_pre"])
    dx, du, dgate, dw_post, dw_pre = sdgp.sdgp_block_norm_bwd(t["dy"], t["dh"], y, stats, t["u"], t["gate"], t["w_post"], t["w_pre"])
    per = rows // gate
    post, pre, sizes = 0.0, 0.0, 0.0
    for g in range(gate):
        gates = []
        for cut in (slice(g * per, g * per + per // 2), slice(g * per + per // 2, (g + 1) * per)):
            p = {k: v[cut] for k, v in t.items() if k in ("x", "u", "dy", "dh")}
            one = t["gate"][g].contiguous()
            py, ph, ps = sdgp.sdgp_block_norm(p["x"], p["u"], one, t["w_post"], t["w_pre"])
            assert torch.equal(py, y[cut]) and torch.equal(ph, h[cut]) and torch.equal(ps, stats[:, cut])
            pdx, pdu, pg, p_post, p_pre = sdgp.sdgp_block_norm_bwd(p["dy"], p["dh"], py, ps, p["u"], one, t["w_post"], t["w_pre"])
            assert torch.equal(pdx, dx[cut]) and torch.equal(pdu, du[cut])
            gates.append(f64(pg))
            post, pre = post + f64(p_post), pre + f64(p_pre)
            sizes = sizes + f64((p["dh"].float().abs() * 6 + p["dy"].float().abs()).sum(0)) * 12
        store = 2.0 ** -7 if dtype == torch.bfloat16 else 2 * E
        near(dgate.view(gate, D)[g], gates[0] + gates[1], 2 * E * per * sizes + store * (np.abs(gates[0]) + np.abs(gates[1])), "dgate")
    near(dw_post, post, 2 * E * rows * sizes, "dw_post")
    near(dw_pre, pre, 2 * E * rows * sizes, "dw_pre")


def test_more_elements_than_32_bits_count():
    rows, D = 1100000, 2048
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    x, u, dy, dh = (torch.empty(rows, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(4))
    w = 1 + 0.3 * torch.randn(D, device="cuda", generator=g)
    gate = torch.randn(1, D, device="cuda", generator=g).to(torch.bfloat16)
    y, h, stats = sdgp.sdgp_block_norm(x, u, gate, w, w)
    dx, du, dgate, dw_post, dw_pre = sdgp.sdgp_block_norm_bwd(dy, dh, y, stats, u, gate, w, w)
    for cut in (slice(0, 40), slice(1048560, 1048600), slice(rows - 40, rows)):     # 2^31 elements lie between
        py, ph, ps = sdgp.sdgp_block_norm(x[cut], u[cut], gate, w, w)
        pdx, pdu, *_ = sdgp.sdgp_block_norm_bwd(dy[cut], dh[cut], py, ps, u[cut], gate, w, w)
        for a, b in ((y, py), (h, ph), (dx, pdx), (du, pdu)):
            assert torch.equal(a[cut], b)
    assert torch.isfinite(dw_post).all() and torch.isfinite(dw_pre).all() and torch.isfinite(dgate).all()

"""The sums over rows of the block norms' gradient, for every way in which the rows are cut: many gates of several rows each,
rows in turn where tensors are larger than 128 MB, narrow rows of which a workgroup takes several, none of these.

The reference is the formula in 64 bits, from y as the call stored it, on the GPU in chunks of rows.  Bounds, with e = 2^-24 and
N = D / 64 + 32 (a row's own factor and mean, as in the tests of single rows): a gradient term carries at most 8 N e of its size,
and a sum adds e of the sum of sizes for every addition that a term goes through.  Of those there are at most
    ceil(rows a slab / R) + R      in the slab, whose rows R groups of threads share,
    slabs / 32 + 8 + 5 + gates     where the slabs' sums are added (32 threads a column, eight chains each, a tree; one a gate),
and the slabs are as many as their sums fit into the workspace that the call asks for.  So that the bound says something, it has
to stay below a tenth (of the most rows a fifth) of the sums' own size (root mean square).
"""
import pytest
import torch

import paper_2202_00774_amd as sdgp
from paper_2202_00774_amd import binding

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


def make(rows, D, dtype, gates, seed, block=True, weights=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    def rnd(*s):
        return torch.empty(s, device="cuda", dtype=dtype).normal_(generator=g)
    t = {"x": rnd(rows, D), "u": None, "gate": None, "w_post": None, "w_pre": None, "dy": rnd(rows, D), "dh": rnd(rows, D)}
    if weights:
        t["w_pre"] = 1 + 0.3 * torch.randn(D, device="cuda", generator=g)
    if block:
        t["u"] = rnd(rows, D)
        if weights:
            t["w_post"] = 1 + 0.3 * torch.randn(D, device="cuda", generator=g)
        if gates:
            t["gate"] = rnd(gates, D)
    return t


def near(got, want, bound, what):
    off = ((got.double() - want).abs() - bound).max().item()
    assert off <= 0, (what, off, want.abs().max().item())


def rows_at_once(D, dtype):
    vecs = -(-D // (8 if dtype == BF16 else 4))
    return 16 if vecs <= 16 else 8 if vecs <= 32 else 4 if vecs <= 64 else 2 if vecs <= 128 else 1


def check(t, residual_scale=1.0, eps=1e-6, pre=True, sharp=0.1):
    x, dtype = t["x"], t["x"].dtype
    rows, D = x.shape
    gates = 0 if t["gate"] is None else t["gate"].shape[0]
    per = rows // gates if gates else rows
    w_pre = t["w_pre"] if pre else None
    dh = t["dh"] if pre else None
    y, h, stats = sdgp.sdgp_block_norm(x, t["u"], t["gate"], t["w_post"], w_pre, residual_scale=residual_scale, eps=eps, pre=pre)
    args = (t["dy"], dh, y, stats, t["u"], t["gate"], t["w_post"], w_pre)
    dx, du, dgate, dw_post, dw_pre = got = sdgp.sdgp_block_norm_bwd(*args, residual_scale=residual_scale)

    store, N = (2.0 ** -8 if dtype == BF16 else E), D / 64 + 32
    sums = {k: torch.zeros(2, D, device="cuda", dtype=torch.float64) for k in ("pre", "post")}        # the sum, the sum of sizes
    gate_sums = torch.zeros(2, max(gates, 1), D, device="cuda", dtype=torch.float64)
    wp = 1.0 if t["w_post"] is None else t["w_post"].double()
    wr = 1.0 if w_pre is None else w_pre.double()
    for lo in range(0, rows, max(1, (1 << 24) // D)):
        c = slice(lo, min(rows, lo + max(1, (1 << 24) // D)))
        ys, dY = y[c].double(), t["dy"][c].double()
        size = dY.abs()
        if pre:
            ry = (ys.square().mean(1, keepdim=True) + eps).rsqrt()
            n, d = ys * ry, dh[c].double()
            q = d * wr
            near(h[c], n * wr, (E * N + store) * (n * wr).abs() + 1e-38, "h")
            dY = dY + ry * (q - n * (q * n).mean(1, keepdim=True))
            size = size + ry * (q.abs() + n.abs() * (q * n).abs().mean(1, keepdim=True))
            sums["pre"] += torch.stack([(d * n).sum(0), (d * n).abs().sum(0)])
        f = residual_scale if t["u"] is not None else 1.0
        near(dx[c], f * dY, abs(f) * E * 4 * N * size + store * (f * dY).abs() + 1e-38, "dx")
        if t["u"] is None:
            continue
        us = t["u"][c].double()
        ru = (us.square().mean(1, keepdim=True) + eps).rsqrt()
        a = us * ru
        group = torch.arange(c.start, c.stop, device="cuda") // per
        k = t["gate"].double()[group] if gates else torch.ones_like(a)
        want = residual_scale * x[c].double() + k * a * wp
        near(y[c], want, E * N * ((residual_scale * x[c].double()).abs() + (k * a * wp).abs()) + store * want.abs() + 1e-38, "y")
        q, qs = dY * k * wp, size * (k * wp).abs()
        want = ru * (q - a * (q * a).mean(1, keepdim=True))
        near(du[c], want, ru * E * 8 * N * (qs + a.abs() * (qs * a.abs()).mean(1, keepdim=True)) + store * want.abs() + 1e-38, "du")
        sums["post"] += torch.stack([(dY * k * a).sum(0), (size * (k * a).abs()).sum(0)])
        if gates:
            terms = dY * a * wp, size * (a * wp).abs()
            if per < 4096:
                gate_sums[0].index_add_(0, group, terms[0]), gate_sums[1].index_add_(0, group, terms[1])
                continue
            for g in range(c.start // per, (c.stop - 1) // per + 1):
                part = slice(max(0, g * per - c.start), min(c.stop, (g + 1) * per) - c.start)
                gate_sums[0, g] += terms[0][part].sum(0)
                gate_sums[1, g] += terms[1][part].sum(0)

    need = binding._need("sdgp_block_norm_bwd_workspace", rows, D, gates, binding._dtype_code(x))
    slabs, R = max(1, need // (8 * D)), rows_at_once(D, dtype)      # (of long rows the workspace holds a little more)
    deep = -(-rows // slabs) / R + 1 + R + slabs / 32 + 13 + (gates if gates < 256 else 0) + 8 * N
    for dw, key in ((dw_pre if pre else None, "pre"), (dw_post, "post")):
        if dw is not None:
            bound = E * deep * sums[key][1]
            assert bound.square().mean() < sharp ** 2 * sums[key][0].square().mean()
            near(dw, sums[key][0], bound, "dw_" + key)
    if gates:
        bound = E * (min(per, deep) + 8 * N) * gate_sums[1] + store * gate_sums[0].abs()
        assert bound.square().mean() < sharp ** 2 * gate_sums[0].square().mean()
        near(dgate.view(gates, D), gate_sums[0], bound, "dgate")
    again = sdgp.sdgp_block_norm_bwd(*args, residual_scale=residual_scale)
    for p, q in zip(got, again):
        assert p is None or torch.equal(p, q)
    return slabs


MANY = [(4100, 2050), (6153, 2051), (65600, 2050), (131074, 65537)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [24, 130, 264, 1001])
@pytest.mark.parametrize("rows,gates", MANY)
def test_many_gates_of_several_rows(rows, gates, D, dtype):
    """2048 gates or more of at most 32 rows, or 65536: a slab holds whole gates and finishes them itself."""
    check(make(rows, D, dtype, gates, rows + D), residual_scale=0.75)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [1104, 2560, 5000, 8000, 8200, 16400])
def test_many_gates_of_several_rows_of_every_width(D, dtype):
    """192 to 1024 threads a row, two vectors a thread, rows too long for the registers."""
    D = D // 2 if dtype == F32 else D
    check(make(4100, D, dtype, 2050, D))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [24, 264, 4100, 8200])
def test_many_gates_without_weights_or_the_norm_behind(D, dtype):
    check(make(6153, D, dtype, 2051, D, weights=False))
    check(make(6153, D, dtype, 2051, D + 1), pre=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,gates", [(2100, 700), (4094, 2047), (33 * 2049, 2049), (3000, 1500)])
def test_gates_that_have_slabs_of_their_own(rows, gates, dtype):
    """Fewer than 2048 gates, or more than 32 rows each: the gates' sums are finished behind the slabs."""
    for D in (24, 264, 1001):
        check(make(rows, D, dtype, gates, D))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,gates", [(24, 1), (24, 3), (24, 0), (130, 1), (130, 5), (264, 1), (520, 2), (1001, 1), (1001, 7)])
def test_rows_in_turn(D, gates, dtype):
    """Tensors above 128 MB of narrow and odd rows, several of which a workgroup has in hand."""
    rows = (129 << 20) // (D * (2 if dtype == BF16 else 4)) // 210 * 210
    assert rows * D * (2 if dtype == BF16 else 4) > 128 << 20
    check(make(rows, D, dtype, gates, D), residual_scale=0.5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [24, 130, 1001, 2048])
def test_rows_in_turn_without_a_block_and_with_a_gate_a_row(D, dtype):
    rows = (130 << 20) // (D * (2 if dtype == BF16 else 4))
    check(make(rows, D, dtype, 0, D, block=False))
    check(make(rows, D, dtype, rows, D + 1))


@pytest.mark.parametrize("rows,D,dtype,gates", [(36000, 2048, BF16, 1), (9001, 4097, F32, 1), (18000, 4096, BF16, 4), (140000, 520, BF16, 2)])
def test_sums_of_tensors_larger_than_the_caches(rows, D, dtype, gates):
    slabs = check(make(rows, D, dtype, gates, D))
    assert slabs > 200


def test_sums_of_more_elements_than_32_bits_count():
    check(make(1100000, 2048, BF16, 1, 0), sharp=0.2)      # bounds grow with the rows, such sums with their root

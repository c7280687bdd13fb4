"""rft_linear and rft_linear_bwd against plain float64: both types, every activation, dense and
grouped rows (empty groups, one row, rows of no group, sources out of range), sizes around the
tiles, gradients that are added, streams, graphs and the layer of experts as it is used.

Tolerances.  A product summed over K terms in fp32, in any order, is within (K + 2) 2^-24 times
the sum of the terms' magnitudes (fp32 data; bf16 products are exact in fp32, but the matrix
instruction may truncate where it aligns its terms: 2^-23).  A result is rounded once by at most
half a step.  Activations have slopes of at most 1.13, and fast sigmoids are good to 2^-20."""
import math

import numpy as np
import pytest
import torch

import paper_2505_17826_amd as R
from tests import linear_model as M
from tests.gpu_cases import requires_gpu

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")
CODE = dict(zip(M.ACTS, (R.RFT_ACT_NONE, R.RFT_ACT_SILU, R.RFT_ACT_GELU, R.RFT_ACT_SWIGLU)))
BF, F32 = torch.bfloat16, torch.float32


def half(dt):
    return torch.finfo(dt).eps / 2


def acc_eps(dt):
    return 2.0 ** -23 if dt == BF else 2.0 ** -24


def offsets_of(counts):
    return [0] + list(np.cumsum(counts))


class Case:
    def __init__(self, counts, k, n, act, dt, bias=False, residual=False, spare=0, source=None,
                 div=1, tokens=0, seed=0, scale=1.0):
        g = torch.Generator().manual_seed(seed + 17)
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.offsets, self.act, self.dt = offsets_of(counts), act, dt
        self.rows, self.E, self.k, self.n = self.offsets[-1] + spare, len(counts), k, n
        self.m = n // 2 if act == "swiglu" else n
        self.x = r(tokens or self.rows, k).to(dt)
        self.w = (scale * r(self.E, n, k) / math.sqrt(k)).to(dt)
        self.bias = (0.5 * r(self.E, n)).to(dt) if bias else None
        self.residual = r(self.rows, self.m).to(dt) if residual else None
        self.dy = r(self.rows, self.m).to(dt)
        self.source, self.div = source, div
        self.live = self.offsets[-1]
        self.xr = M.rows_of_x(self.x.double(), source, div, self.rows)

    def groups(self):
        if self.E == 1 and self.source is None and self.live == self.rows:
            return None
        src = None if self.source is None else self.source.to(DEV)
        return R.Groups(torch.tensor(self.offsets, dtype=torch.int32, device=DEV), src, self.div)

    def dev(self, t):
        return None if t is None else t.to(DEV)


def check_forward(c, want_z=True):
    d = c.dev
    y0 = torch.full((c.rows, c.m), 7.0, dtype=c.dt, device=DEV)
    z0 = torch.full((c.rows, c.n), 7.0, dtype=c.dt, device=DEV)
    y, z = R.rft_linear(d(c.x), d(c.w), bias=d(c.bias), act=CODE[c.act], residual=d(c.residual),
                        groups=c.groups(), out=y0, z=z0 if want_z else None)
    y = y.cpu().double()
    ry, rz, mag = M.forward(c.xr, c.w.double(), None if c.bias is None else c.bias.double(), c.act,
                            None if c.residual is None else c.residual.double(), c.offsets)
    live = slice(0, c.live)
    tz = (c.k + 3) * acc_eps(c.dt) * mag[live]
    if want_z:
        zz = z.cpu().double()
        assert ((zz[live] - rz[live]).abs() <= tz + half(c.dt) * (rz[live].abs() + tz)).all()
        assert (zz[c.live:] == 7).all()
    slack = 2.0 ** -20 if c.dt == BF else 2.0 ** -21  # sigmoid, erfc, exp: a few ulps
    a = M.value(rz[live], c.act)
    if c.act == "swiglu":
        g, u = rz[live, :c.m], rz[live, c.m:]
        ty = 1.13 * tz[:, :c.m] * (u.abs() + tz[:, c.m:]) + g.abs() * tz[:, c.m:] + slack * (g * u).abs()
    else:
        ty = (1.0 if c.act == "none" else 1.13) * tz + (0 if c.act == "none" else slack) * rz[live].abs()
    ty = ty + 2.0 ** -23 * (a.abs() + ry[live].abs())
    tol = ty + half(c.dt) * (ry[live].abs() + ty)
    err = (y[live] - ry[live]).abs()
    assert (err <= tol).all(), float((err / tol).max())
    assert (y[c.live:] == 7).all()
    return rz


def check_backward(c, z=None, dw_dtype=None, accumulate=False, want_db=True):
    d = c.dev
    if z is None and c.act != "none":
        z = torch.randn(c.rows, c.n, generator=torch.Generator().manual_seed(5)).to(c.dt)
    dw_dtype = dw_dtype or c.dt
    g0 = torch.Generator().manual_seed(9)
    dw0, db0 = torch.randn(c.w.shape, generator=g0), torch.randn(c.E, c.n, generator=g0)
    dx0 = torch.full((c.rows, c.k), 7.0, dtype=c.dt, device=DEV)
    dx, dw, db = R.rft_linear_bwd(
        d(c.dy), d(c.x), d(c.w), z=d(z), act=CODE[c.act], groups=c.groups(), d_x=dx0,
        d_weight=d(dw0).to(dw_dtype).contiguous(), d_bias=d(db0) if want_db else None,
        accumulate=accumulate)
    rx, rw, rb, dz, mx, mw, mb = M.backward(
        c.dy.double(), None if z is None else z.double(), c.xr, c.w.double(), c.act, c.offsets)
    live = slice(0, c.live)
    # dz: a product of up to three factors, then rounded for the products (not with act none)
    s = 2.0 ** -19 if c.act != "none" else 0.0
    rounded = half(BF) if c.dt == BF and c.act != "none" else 0.0
    if c.act in ("silu", "gelu", "swiglu"):
        # a slope is a sum of terms of up to |z| and 1: its error is absolute
        zz = z.double()[live]
        gz = zz[:, :c.m] if c.act == "swiglu" else zz
        amp = c.dy.double()[live].abs() * (1 + gz.abs())
        if c.act == "swiglu":
            amp = torch.cat([amp * zz[:, c.m:].abs(), amp], 1)
        ed = s * amp + rounded * (dz[live].abs() + s * amp)
    else:
        ed = torch.zeros_like(dz[live])
    full = torch.zeros_like(dz)
    full[live] = ed
    w64, x64 = c.w.double().abs(), c.xr.abs()
    ex, ew, eb = torch.zeros_like(rx), torch.zeros_like(rw), torch.zeros_like(rb)
    for e in range(c.E):
        a, b = c.offsets[e], c.offsets[e + 1]
        ex[a:b] = full[a:b] @ w64[e]
        ew[e] = full[a:b].T @ x64[a:b]
        eb[e] = s / max(s, 1e-300) * full[a:b].sum(0) if s else 0
    tx = ex[live] + (c.n + 3) * acc_eps(c.dt) * (mx[live] + ex[live])
    x = dx.cpu().double()
    err, tol = (x[live] - rx[live]).abs(), tx + half(c.dt) * (rx[live].abs() + tx)
    assert (err <= tol).all(), ("d_x", float((err / tol).max()))
    assert (x[c.live:] == 7).all()
    most = max([b - a for a, b in zip(c.offsets, c.offsets[1:])])
    tw = ew + (most + 3) * acc_eps(c.dt) * (mw + ew)
    rw = rw + dw0.double() if accumulate else rw
    err, tol = (dw.cpu().double() - rw).abs(), tw + half(dw_dtype) * (rw.abs() + tw) + 1e-30
    assert (err <= tol).all(), ("d_weight", float((err / tol).max()))
    if want_db:
        rb = rb + db0.double() if accumulate else rb
        err, tol = (db.cpu().double() - rb).abs(), eb + (most + 8) * 2.0 ** -24 * (mb + eb) + half(F32) * rb.abs() + 1e-30
        assert (err <= tol).all(), ("d_bias", float((err / tol).max()))
    return dx, dw, db


GROUPS = [  # counts, rows of no group behind them
    ([1], 0), ([5], 0), ([130], 0), ([257], 3), ([0, 3, 0, 1, 129, 0], 0), ([64] * 9, 5),
    ([0, 0, 0], 4), ([300, 1, 17], 0)]


@pytest.mark.parametrize("dt", (BF, F32))
@pytest.mark.parametrize("act", M.ACTS)
@pytest.mark.parametrize("counts,spare", GROUPS)
def test_forward(counts, spare, act, dt):
    k, n = (72, 208) if dt == BF else (71, 206)
    check_forward(Case(counts, k, n, act, dt, bias=True, residual=True, spare=spare, seed=len(counts)))


SIZES = [(8, 16), (64, 16), (128, 256), (136, 272), (520, 1040), (1000, 48)]


@pytest.mark.parametrize("dt", (BF, F32))
@pytest.mark.parametrize("k,n", SIZES)
def test_forward_sizes(k, n, dt):
    if dt == F32:
        k, n = k + 1, n + 2
    for act in ("none", "swiglu"):
        check_forward(Case([37, 0, 140], k, n, act, dt, seed=k), want_z=act == "swiglu")


@pytest.mark.parametrize("dt", (BF, F32))
@pytest.mark.parametrize("n", (1, 3, 16, 64))
def test_few_rows(n, dt):
    """Rows of single tokens: every count of rows of an expert from 0 to 40."""
    if dt == BF:
        n = max(16, n)
    counts = [0, 1, 2, 3, 0, 7, 8, 15, 16, 17, 31, 32, 33, 40]
    check_forward(Case(counts, 264 if dt == BF else 263, 2 * n, "swiglu", dt, bias=True, seed=n))
    check_forward(Case([1], 1032, 48 * n, "none", dt, residual=True, seed=n))


def test_large_tiles():
    """Enough tiles for the larger tile, ragged at every edge."""
    c = Case([700, 0, 1, 2085, 3], 328, 4168, "none", BF, bias=True, spare=2, seed=3)
    check_forward(c)
    check_backward(c, dw_dtype=F32)
    c = Case([1111, 700], 200, 4112, "swiglu", BF, seed=4)
    check_forward(c)
    check_backward(c)


@pytest.mark.parametrize("act", ("none", "swiglu"))
@pytest.mark.parametrize("rows,k,n", [(4352, 4096, 4096), (4100, 4104, 4352), (2100, 8200, 2064)])
def test_tail_in_slices(rows, k, n, act):
    """Dense layers whose last tiles are cut along the summed index, against float64 on the GPU."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    x, w, b = r(rows, k).to(BF), (r(n, k) / math.sqrt(k)).to(BF), r(n).to(BF)
    m = n // 2 if act == "swiglu" else n
    res, dy = r(rows, m).to(BF), r(rows, m).to(BF)
    y, z = R.rft_linear(x, w, bias=b, act=CODE[act], residual=res, want_z=True)
    x6, w6 = x.double(), w.double()
    want = x6 @ w6.T.contiguous() + b.double()
    eps = 2.0 ** -23
    tz = (k + 3) * eps * (x6.abs() @ w6.abs().T.contiguous() + b.double().abs())
    assert bool(((z.double() - want).abs() <= tz + half(BF) * (want.abs() + tz)).all())
    # y by its own rounding and z's error through slopes of at most 1.13 |u| and |silu(g)|
    a = M.value(want, act)
    if act == "swiglu":
        u = want[:, m:].abs()
        ty = 1.13 * tz[:, :m] * (u + tz[:, m:]) + want[:, :m].abs() * tz[:, m:] + 2.0 ** -20 * a.abs()
    else:
        ty = tz
    yw = a + res.double()
    ty = ty + 2.0 ** -22 * (a.abs() + yw.abs())
    assert bool(((y.double() - yw).abs() <= ty + half(BF) * (yw.abs() + ty)).all())
    if act != "none":
        return
    dw0 = r(n, k)
    dx, dw, _ = R.rft_linear_bwd(dy, x, w, d_weight=dw0.clone(), accumulate=True)
    d6 = dy.double()
    want, t = d6 @ w6, (n + 3) * eps * (d6.abs() @ w6.abs())
    assert bool(((dx.double() - want).abs() <= t + half(BF) * (want.abs() + t)).all())
    dT = d6.T.contiguous()
    want, t = dT @ x6 + dw0.double(), (rows + 4) * eps * (dT.abs() @ x6.abs() + dw0.double().abs())
    assert bool(((dw.double() - want).abs() <= t).all())
    only = R.rft_linear_bwd(dy, x, w, want_dx=False)[1]
    want, t = dT @ x6, (rows + 3) * eps * (dT.abs() @ x6.abs())
    assert bool(((only.double() - want).abs() <= t + half(BF) * (want.abs() + t)).all())


@pytest.mark.parametrize("dt", (BF, F32))
@pytest.mark.parametrize("act", M.ACTS)
@pytest.mark.parametrize("counts,spare", GROUPS)
def test_backward(counts, spare, act, dt):
    k, n = (72, 208) if dt == BF else (71, 206)
    check_backward(Case(counts, k, n, act, dt, spare=spare, seed=len(counts)))


@pytest.mark.parametrize("dt", (BF, F32))
def test_backward_added(dt):
    c = Case([40, 0, 9], 136, 64, "silu", dt, spare=1, seed=8)
    check_backward(c, dw_dtype=F32, accumulate=True)
    c = Case([5000], 40, 64, "none", dt, seed=9)  # slices of a long group's rows
    check_backward(c, dw_dtype=F32, accumulate=True)
    check_backward(c, dw_dtype=dt)


@pytest.mark.parametrize("dt", (BF, F32))
@pytest.mark.parametrize("k,n", SIZES)
def test_backward_sizes(k, n, dt):
    if dt == F32:
        k, n = k + 1, n + 2
    check_backward(Case([37, 0, 140], k, n, "none", dt, seed=k), dw_dtype=F32)


def test_many_tiles_of_sources():
    """Several tiles per block of both tile sizes, each with its own rows of the tokens."""
    g = torch.Generator().manual_seed(13)
    for counts, k, n in (([300, 0, 70, 513], 1032, 4104), ([100] * 40, 264, 528)):
        rows, tokens, div = sum(counts), 61, 3
        source = torch.randint(0, tokens * div, (rows,), generator=g, dtype=torch.int32)
        c = Case(counts, k, n, "none", BF, source=source, div=div, tokens=tokens, seed=k)
        check_forward(c, want_z=False)
        check_backward(c, dw_dtype=F32)


@pytest.mark.parametrize("dt", (BF, F32))
def test_sources(dt):
    """Rows taken from the tokens by slots, some of them no row of x."""
    g = torch.Generator().manual_seed(3)
    counts, div, tokens = [200, 3, 0, 61], 4, 50
    rows = sum(counts) + 6
    source = torch.randint(0, tokens * div, (rows,), generator=g, dtype=torch.int32)
    source[5], source[100], source[201] = -1, tokens * div, 2 ** 31 - 1
    for act in ("none", "swiglu"):
        c = Case(counts, 136, 160, act, dt, spare=6, source=source, div=div, tokens=tokens, seed=11)
        check_forward(c)
        check_backward(c, dw_dtype=F32 if act == "none" else None)


@pytest.mark.parametrize("dt", (BF, F32))
def test_values_at_the_ends(dt):
    """Large, infinite and NaN pre-activations, forward and backward; other rows are untouched."""
    big = torch.tensor([0.0, -0.0, 1e-30, 20.0, -20.0, 100.0, -100.0, 3e38, -3e38, math.inf, -math.inf])
    n = 16
    z = torch.zeros(len(big) + 1, n)
    z[:len(big)] = big[:, None]
    z[-1] = math.nan
    z = z.to(dt)
    dy = torch.ones(z.shape[0], n, dtype=dt)
    x, w = torch.zeros(z.shape[0], 8, dtype=dt), torch.zeros(n, 8, dtype=dt)
    for act, lim in (("silu", R.RFT_ACT_SILU), ("gelu", R.RFT_ACT_GELU)):
        db = R.rft_linear_bwd(dy.to(DEV), x.to(DEV), w.to(DEV), z=z.to(DEV), act=lim, want_db=True,
                              groups=R.Groups(torch.tensor([0, len(big)], dtype=torch.int32, device=DEV)))[2]
        zz = z[:len(big)].double().clamp(-700, 700)
        want = M.slopes(zz, act)[0].sum(0)
        assert ((db.cpu().double() - want).abs() <= 1e-5).all(), act
        # forward by a bias that is z
        y, _ = R.rft_linear(torch.zeros(len(big), 8, dtype=dt, device=DEV),
                            torch.zeros(len(big), n, 8, dtype=dt, device=DEV), bias=z[:len(big)].to(DEV), act=lim,
                            groups=R.Groups(torch.arange(len(big) + 1, dtype=torch.int32, device=DEV)))
        want = M.value(z[:len(big)].double(), act).nan_to_num(0.0, math.inf, -math.inf) if act == "silu" else \
            torch.where(z[:len(big)] == -math.inf, torch.zeros_like(zz), M.value(z[:len(big)].double(), act))
        y = y.cpu().double()
        inf = torch.isinf(want) | (want > torch.finfo(dt).max)
        assert (y[inf] > 3e38).all()
        # silu below x = -88.7: exp(-x) passes fp32's range and the sigmoid is 0, where it is less
        # than 2^-128 and |x| sigmoid(x), falling from there, less than 88.8 2^-128 < 2^-121
        tol = (half(dt) + 2.0 ** -20) * want[~inf].abs() + 2.0 ** -121
        assert bool(((y - want)[~inf].abs() <= tol).all()), act
    # a NaN or inf in one row of x stays in its row
    x = torch.randn(40, 64, generator=torch.Generator().manual_seed(1)).to(dt)
    x[7, 3], x[20, 0] = math.nan, math.inf
    w = torch.ones(16, 64, dtype=dt)
    y = R.rft_linear(x.to(DEV), w.to(DEV))[0].cpu()
    fine = torch.isfinite(y.double()).all(1)
    assert not fine[7] and not fine[20] and int(fine.sum()) == 38


def test_no_rows_and_no_tokens():
    w = torch.randn(3, 16, 8, device=DEV)
    off = torch.zeros(4, dtype=torch.int32, device=DEV)
    y, _ = R.rft_linear(torch.empty(0, 8, device=DEV), w, groups=R.Groups(off))
    assert y.shape == (0, 16)
    dx, dw, db = R.rft_linear_bwd(torch.empty(0, 16, device=DEV), torch.empty(0, 8, device=DEV), w,
                                  groups=R.Groups(off), want_db=True)
    assert dx.shape == (0, 8) and not dw.any() and not db.any()


@pytest.mark.parametrize("dt", (BF, F32))
def test_rows_before_the_first_group(dt):
    c = Case([15, 0, 13], 72, 80, "silu", dt, seed=3)
    x, dy = torch.cat([torch.full((5, 72), math.nan, dtype=dt), c.x]), torch.cat([torch.full((5, 80), math.nan, dtype=dt), c.dy])
    g = R.Groups(torch.tensor([5, 20, 20, 33], dtype=torch.int32, device=DEV))
    y0 = torch.full((33, 80), 7.0, dtype=dt, device=DEV)
    y, z = R.rft_linear(x.to(DEV), c.w.to(DEV), act=R.RFT_ACT_SILU, groups=g, out=y0, want_z=True)
    y1, z1 = R.rft_linear(c.x.to(DEV), c.w.to(DEV), act=R.RFT_ACT_SILU, groups=c.groups(), want_z=True)
    assert torch.equal(y[5:], y1) and bool((y[:5] == 7).all())
    d0 = torch.full((33, 72), 7.0, dtype=dt, device=DEV)
    a = R.rft_linear_bwd(dy.to(DEV), x.to(DEV), c.w.to(DEV), z=z, act=R.RFT_ACT_SILU, groups=g, d_x=d0, want_db=True)
    b = R.rft_linear_bwd(c.dy.to(DEV), c.x.to(DEV), c.w.to(DEV), z=z1, act=R.RFT_ACT_SILU, groups=c.groups(), want_db=True)
    assert torch.equal(a[0][5:], b[0]) and bool((a[0][:5] == 7).all())
    # the rows of a group are summed in the same order wherever they lie
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    only = R.rft_linear_bwd(dy.to(DEV), x.to(DEV), c.w.to(DEV), z=z, act=R.RFT_ACT_SILU, groups=g)[1]
    assert torch.equal(only, b[1])


@pytest.mark.parametrize("dt", (BF, F32))
def test_one_group_with_a_source(dt):
    """A dense layer of chosen rows; of no rows at all, where the bias is left."""
    g = torch.Generator().manual_seed(4)
    x, w, b = (torch.randn(*s, generator=g).to(dt) for s in ((30, 64), (48, 64), (48,)))
    for count in (7, 300):
        src = torch.randint(0, 30, (count,), generator=g, dtype=torch.int32)
        groups = R.Groups(None, src.to(DEV))
        y, _ = R.rft_linear(x.to(DEV), w.to(DEV), groups=groups)
        same, _ = R.rft_linear(x[src.long()].to(DEV), w.to(DEV))
        assert torch.equal(y, same)
        dw = R.rft_linear_bwd(y, x.to(DEV), w.to(DEV), groups=groups, want_dx=False)[1]
        assert torch.equal(dw, R.rft_linear_bwd(y, x[src.long()].to(DEV), w.to(DEV), want_dx=False)[1])
        none = torch.empty(0, 64, dtype=dt, device=DEV)
        y, _ = R.rft_linear(none, w.to(DEV), bias=b.to(DEV), groups=groups)
        assert torch.equal(y.cpu(), b.expand(count, 48))
        assert not R.rft_linear_bwd(y, none, w.to(DEV), groups=groups, want_dx=False)[1].any()


def test_offsets_that_are_not_valid_stay_inside():
    """Offsets that decrease or leave the rows: unspecified values, but only the rows' places."""
    for dt in (BF, F32):
        x, w = torch.randn(64, 64, device=DEV).to(dt), torch.randn(4, 64, 64, device=DEV).to(dt)
        for off in ([0, 1000, 3, 64, 64], [-5, 10, 5, 7, 2 ** 31 - 1], [64, 0, 64, 0, 64]):
            g = R.Groups(torch.tensor(off, dtype=torch.int32, device=DEV))
            buf = torch.full((66 * 64,), 7.0, dtype=dt, device=DEV)
            R.rft_linear(x, w, groups=g, out=buf[64:65 * 64].view(64, 64))
            R.rft_linear_bwd(x, x, w, groups=g, d_x=buf[64:65 * 64].view(64, 64))
            assert (buf[:64] == 7).all() and (buf[65 * 64:] == 7).all()


def test_gradient_by_differences():
    """fp32: the slope of <dy, y> along random directions of x, w and bias."""
    c = Case([9, 0, 20], 33, 26, "swiglu", F32, bias=True, seed=21)
    d = c.dev
    g = torch.Generator().manual_seed(2)
    dirs = [torch.randn(t.shape, generator=g) for t in (c.x, c.w, c.bias)]
    _, z = R.rft_linear(d(c.x), d(c.w), bias=d(c.bias), act=CODE[c.act], groups=c.groups(), want_z=True)
    dx, dw, db = R.rft_linear_bwd(d(c.dy), d(c.x), d(c.w), z=z, act=CODE[c.act], groups=c.groups(),
                                  want_db=True)
    h = 2.0 ** -8
    for i, grad in enumerate((dx, dw, db)):
        def loss(t):
            p = [q + (t * dirs[i] if j == i else 0) for j, q in enumerate((c.x, c.w, c.bias))]
            y, _ = R.rft_linear(d(p[0]), d(p[1]), bias=d(p[2]), act=CODE[c.act], groups=c.groups())
            return (y.cpu().double() * c.dy.double()).sum()
        # fourth order: h^4 times a fifth derivative of a few thousands of terms of size 1; the
        # fp32 rounding of each y (2^-22 of a few units, random signs over 377) over h
        slope = (8 * (loss(h) - loss(-h)) - (loss(2 * h) - loss(-2 * h))) / (12 * h)
        want = (grad.cpu().double() * dirs[i].double()).sum()
        size = (grad.cpu().double().norm() * dirs[i].double().norm())
        assert abs(slope - want) <= 1e-3 * size, (i, float(slope), float(want))


def test_layer_of_experts():
    """The run of entry points as it is used: router, order, up and down projections, sum; and
    its backward, against float64 throughout."""
    T, E, k, d, f = 150, 12, 3, 72, 40
    g = torch.Generator().manual_seed(31)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x, wu, wd = r(T, d), r(E, 2 * f, d) / math.sqrt(d), r(E, d, f) / math.sqrt(f)
    wr, do = r(E, d) / math.sqrt(d), r(T, d)
    mask = (torch.rand(T, generator=g) < 0.8).to(torch.uint8)
    dv = lambda t: t.to(DEV)  # noqa: E731
    tok = R.Tokens(torch.tensor([0, 70, T], dtype=torch.int32, device=DEV), dv(mask))
    prm = R.router_params(E, k, norm_topk=True)
    X, WU, WD, WR, DO = map(dv, (x, wu, wd, wr, do))
    logits, _ = R.rft_linear(X, WR)
    fwd = R.rft_router_fwd(tok, logits, prm)
    o = R.rft_expert_sort(fwd.expert_ids, E)
    up, rows = o.groups(gather=True), o.groups()
    h, z = R.rft_linear(X, WU, act=R.RFT_ACT_SWIGLU, groups=up, want_z=True)
    y, _ = R.rft_linear(h, WD, groups=rows)
    out = R.rft_expert_combine(o, y, gates=fwd.gates, residual=X)
    d_y, d_gates = R.rft_expert_combine_bwd(o, DO, y, gates=fwd.gates)
    d_h, d_wd, _ = R.rft_linear_bwd(d_y, h, WD, groups=rows)
    d_rows, d_wu, _ = R.rft_linear_bwd(d_h, X, WU, z=z, act=R.RFT_ACT_SWIGLU, groups=up)
    d_logits = R.rft_router_bwd(tok, logits, prm, fwd, d_gates=d_gates)
    d_x, d_wr, _ = R.rft_linear_bwd(d_logits, X, WR)
    d_x = R.rft_expert_combine(o, d_rows, residual=d_x) + DO

    leaves = [t.double().requires_grad_() for t in (x, wu, wd, wr)]
    x6, wu6, wd6, wr6 = leaves
    ids = fwd.expert_ids.cpu().long()
    p = torch.softmax(x6 @ wr6.T, 1)
    live = mask.bool()
    s = torch.gather(p, 1, ids.clamp(min=0))
    s = s / s.sum(1, keepdim=True)
    zz = torch.einsum("td,tkfd->tkf", x6, wu6[ids.clamp(min=0)])
    hh = torch.nn.functional.silu(zz[..., :f]) * zz[..., f:]
    yy = torch.einsum("tkf,tkdf->tkd", hh, wd6[ids.clamp(min=0)])
    want = x6 + torch.where(live[:, None], (s[..., None] * yy).sum(1), torch.zeros(()).double())
    (want * do.double()).sum().backward()
    near = lambda a, b: float((a.cpu().double() - b).norm() / b.norm())  # noqa: E731
    # a handful of fp32 products in a row, each within sqrt(100) 2^-24 of its norm
    assert near(out, want.detach()) < 2e-6
    for got, leaf in ((d_x, x6), (d_wu, wu6), (d_wd, wd6), (d_wr, wr6)):
        assert near(got, leaf.grad) < 1e-5


def test_streams_graphs_and_repeats():
    """The same bits from another stream, from a second call, and from a captured graph replayed
    between eager calls, in workspaces of its own."""
    c = Case([100, 0, 31, 400], 136, 96, "swiglu", BF, seed=6)
    d = c.dev
    x, w, dy, groups = d(c.x), d(c.w), d(c.dy), c.groups()

    def call(stream=None):
        y, z = R.rft_linear(x, w, act=CODE[c.act], groups=groups, want_z=True, stream=stream)
        dx, dw, db = R.rft_linear_bwd(dy, x, w, z=z, act=CODE[c.act], groups=groups, want_db=True,
                                      stream=stream)
        return y, z, dx, dw, db

    first = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = call(side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, other):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for i in range(3):
        for t in held:
            t.zero_()
        graph.replay()
        again = call()
        torch.cuda.synchronize()
        for a, b, e in zip(first, held, again):
            assert torch.equal(a, b) and torch.equal(a, e), i
        x.mul_(-1) if i == 0 else None
        if i == 0:
            first = call()


def test_tail_of_chosen_rows_in_a_graph():
    """One group of chosen rows whose last tiles are cut (272 tiles of 256 x 256): the bits of the rows
    gathered first, eager and from a graph replayed with other rows."""
    rows, k, n = 4352, 4096, 4096
    g = torch.Generator(device=DEV).manual_seed(11)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV).to(BF)  # noqa: E731
    x, w, dy = r(1500, k), (r(n, k) / 64), r(rows, n)
    src = torch.randint(0, 1500, (rows,), generator=g, dtype=torch.int32, device=DEV)
    groups = R.Groups(None, src)

    def call():
        y, _ = R.rft_linear(x, w, groups=groups)
        dx, dw, _ = R.rft_linear_bwd(dy, x, w, groups=groups)
        return y, dx, dw

    def gathered():
        rows_ = x[src.long()]
        y, _ = R.rft_linear(rows_, w)
        dx, dw, _ = R.rft_linear_bwd(dy, rows_, w)
        return y, dx, dw

    for a, b in zip(call(), gathered()):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for i in range(3):
        src.copy_(torch.randint(0, 1500, (rows,), generator=g, dtype=torch.int32, device=DEV))
        for t in held:
            t.zero_()
        graph.replay()
        want = gathered()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b), i


def test_past_32_bits():
    """x of more than 2^32 bytes, dense and in groups: rows at its end, and the sums over all of it."""
    rows, k, n = 1_150_000, 2048, 16
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(rows, k, generator=g, device=DEV, dtype=BF)
    w = (torch.randn(2, n, k, generator=g, device=DEV) / math.sqrt(k)).to(BF)
    dy = torch.randn(rows, n, generator=g, device=DEV).to(BF)
    cut = 1_100_001
    groups = R.Groups(torch.tensor([0, cut, rows], dtype=torch.int32, device=DEV))
    y, _ = R.rft_linear(x, w, groups=groups)
    dx, dw, db = R.rft_linear_bwd(dy, x, w, groups=groups, dw_dtype=F32, want_db=True)
    for a, b, e in ((0, 300, 0), (cut - 300, cut, 0), (cut, cut + 300, 1), (rows - 300, rows, 1)):
        x6, w6, d6 = x[a:b].double(), w[e].double(), dy[a:b].double()
        for got, want, mag, terms in ((y[a:b], x6 @ w6.T.contiguous(), x6.abs() @ w6.abs().T.contiguous(), k),
                                      (dx[a:b], d6 @ w6, d6.abs() @ w6.abs(), n)):
            t = (terms + 3) * 2.0 ** -23 * mag
            assert bool(((got.double() - want).abs() <= t + half(BF) * (want.abs() + t)).all()), (a, e)
    for e, (a, b) in enumerate(((0, cut), (cut, rows))):
        want, mag = torch.zeros(n, k, dtype=torch.float64, device=DEV), torch.zeros((), device=DEV)
        for i in range(a, b, 100_000):
            j = min(b, i + 100_000)
            want += dy[i:j].double().T.contiguous() @ x[i:j].double()
        # 2^20 products of unit size summed in fp32: sums of up to a few 2^10, whose roundings (2^-23
        # of them, 2^15 of the matrix instruction) add up like sqrt(2^15) at random; ten times that
        assert float((dw[e].double() - want).abs().max()) <= 10 * 2 ** 12 * 2.0 ** -23 * 2 ** 7.5
        s = dy[a:b].double().sum(0)
        assert bool(((db[e].double() - s).abs() <= 2.0 ** -23 * dy[a:b].double().abs().sum(0)).all())

"""Values at the ends of the types and arrays past 32 bits, for the grouped linear layers.

NaN and infinite pre-activations in rows that count, every activation (swiglu with gates and up values
there), each in its own place and no other; dz itself through an identity weight.  Whole numbers through
arrays of more than 2^32 bytes, dense and in groups: every sum is a whole number below 2^24, so results
are exact and a row that is lost, doubled or taken from elsewhere shows."""
import math

import pytest
import torch

import paper_2505_17826_amd as R
from tests import linear_model as M
from tests.gpu_cases import requires_gpu

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")
BF, F32 = torch.bfloat16, torch.float32
CODE = dict(zip(M.ACTS, (R.RFT_ACT_NONE, R.RFT_ACT_SILU, R.RFT_ACT_GELU, R.RFT_ACT_SWIGLU)))
ENDS = [0.0, -0.0, 1e-30, 1.0, -1.0, 20.0, -20.0, 100.0, -100.0, 3e38, -3e38, math.inf, -math.inf, math.nan]
N = 16


def pre(act, dt):
    """A row per value: z of N columns with the value in column 3 (swiglu: of the gate; the up half is
    1.5 there), 0.5 elsewhere; and the columns of y."""
    n = 2 * N if act == "swiglu" else N
    z = torch.full((len(ENDS), n), 0.5)
    z[:, 3] = torch.tensor(ENDS)
    if act == "swiglu":
        z[:, N + 3] = 1.5
    return z.to(dt)


def limits(z, act):
    """Value and slopes in 64 bits, with the limits at infinities."""
    z = z.double()
    if act == "none":
        return z, (torch.ones_like(z),)
    g = z[:, :N] if act == "swiglu" else z
    c = g.clamp(-700, 700)
    s = M.slopes(c, "gelu" if act == "gelu" else "silu")[0]
    v = M.value(g, "gelu" if act == "gelu" else "silu")
    v = torch.where(g == -math.inf, torch.zeros_like(v), torch.where(g == math.inf, g, v))
    if act == "swiglu":
        return v * z[:, N:], (z[:, N:] * s, v)
    return v, (s,)


def close(got, want, dt, tiny, parts=0.0):
    """tiny: 2^-121 where silu's sigmoid leaves fp32's range below -88.7 (times the factors here), or
    what a slope, a sum of terms, is off; parts: what two bf16 parts leave of a value."""
    got = got.cpu().double()
    assert torch.equal(got.isnan(), want.isnan())
    inf = want.abs() > torch.finfo(dt).max
    assert torch.equal(got[inf], torch.where(want[inf] > 0, math.inf, -math.inf).double())
    fine = ~inf & ~want.isnan()
    tol = (torch.finfo(dt).eps / 2 + 2.0 ** -18 + parts) * want[fine].abs() + tiny
    assert bool(((got - want)[fine].abs() <= tol).all())


@pytest.mark.parametrize("few", (True, False))
@pytest.mark.parametrize("dt", (BF, F32))
@pytest.mark.parametrize("act", M.ACTS)
def test_forward(act, dt, few):
    """By a bias per group of one row that is z; few False: groups of 150 equal rows, in tiles."""
    z = pre(act, dt)
    E, n = z.shape
    each = 1 if few else 150
    off = (torch.arange(E + 1) * each).int().to(DEV)
    x, w = torch.zeros(E * each, 8, dtype=dt, device=DEV), torch.zeros(E, n, 8, dtype=dt, device=DEV)
    y, kept = R.rft_linear(x, w, bias=z.to(DEV), act=CODE[act], groups=R.Groups(off), want_z=True)
    want = limits(z, act)[0].repeat_interleave(each, 0)
    close(y, want, dt, 2.0 ** -120)
    zz = z.repeat_interleave(each, 0)
    assert torch.equal(kept.cpu().isnan(), zz.isnan())
    assert torch.equal(kept.cpu().nan_to_num(7.0), zz.nan_to_num(7.0))


@pytest.mark.parametrize("dt", (BF, F32))
@pytest.mark.parametrize("act", M.ACTS)
def test_bias_gradient(act, dt):
    """dz of one row per group."""
    z = pre(act, dt)
    E, n = z.shape
    off = torch.arange(E + 1, dtype=torch.int32, device=DEV)
    dy = torch.full((E, N), 0.75, dtype=dt, device=DEV)
    x, w = torch.zeros(E, 8, dtype=dt, device=DEV), torch.zeros(E, n, 8, dtype=dt, device=DEV)
    db = R.rft_linear_bwd(dy, x, w, z=z.to(DEV), act=CODE[act], groups=R.Groups(off), want_dx=False, want_dw=False,
                          want_db=True)[2]
    # slopes are sums of terms of up to 1 and more: 2^-18 of 0.75 1.5 at most
    want = torch.cat([0.75 * s for s in limits(z, act)[1]], 1)
    close(db, want, F32, 2.0 ** -18 * 1.125)


@pytest.mark.parametrize("dt", (BF, F32))
@pytest.mark.parametrize("act", M.ACTS)
def test_dz_through_an_identity(act, dt):
    """d_x with an identity weight is dz; d_weight with an identity for x too.  Rows with an infinite or NaN
    dz are NaN in d_x where others take part (0 times them), and stay in their row."""
    z = pre(act, dt)
    rows, n = z.shape
    dy = torch.full((rows, N), 0.75, dtype=dt, device=DEV)
    want = torch.cat([0.75 * s for s in limits(z, act)[1]], 1)
    fine = (want.abs() <= torch.finfo(dt).max).all(1)
    assert int(fine.sum()) >= rows - 3
    eye = torch.eye(n, dtype=dt, device=DEV)
    x = torch.zeros(rows, n, dtype=dt, device=DEV)
    dx = R.rft_linear_bwd(dy, x, eye, z=z.to(DEV), act=CODE[act], want_dw=False)[0].cpu()
    assert not torch.isfinite(dx[~fine]).all(1).any()
    # bf16: dz is rounded, and then the result, which is the same value
    close(dx[fine], want[fine], dt, 2.0 ** -18 * 1.125)
    rows8 = [i for i in range(rows) if fine[i]][:8]
    eye8 = torch.eye(8, dtype=dt, device=DEV)
    for dwt in {dt, F32}:
        dw = R.rft_linear_bwd(dy[:8], eye8, torch.zeros(n, 8, dtype=dt, device=DEV), z=z[rows8].to(DEV), act=CODE[act],
                              want_dx=False, dw_dtype=dwt)[1]
        close(dw.t(), want[rows8], dwt, 2.0 ** -18 * 1.125, 2.0 ** -16 if (dt, dwt) == (BF, F32) else 0.0)


def whole(g, rows, cols, dt):
    """-1, 0 and 1."""
    out = torch.empty(rows, cols, dtype=dt, device=DEV)
    for a in range(0, rows, 100_000):
        b = min(rows, a + 100_000)
        out[a:b] = torch.randint(-1, 2, (b - a, cols), generator=g, device=DEV, dtype=torch.int8).to(dt)
    return out


@pytest.mark.parametrize("cut", (None, 1_100_001))
@pytest.mark.parametrize("dt,rows,k,n", [(BF, 1_150_000, 2048, 16), (BF, 1_150_000, 16, 2048), (F32, 560_000, 2048, 16),
                                         (F32, 560_000, 16, 2048)])
def test_whole_numbers_past_32_bits(dt, rows, k, n, cut):
    g = torch.Generator(device=DEV).manual_seed(rows + k)
    cut = cut if cut is None else min(cut, rows - 40_001)
    E = 1 if cut is None else 2
    x, dy = whole(g, rows, k, dt), whole(g, rows, n, dt)
    w = whole(g, E * n, k, dt).view(E, n, k)
    groups = None if cut is None else R.Groups(torch.tensor([0, cut, rows], dtype=torch.int32, device=DEV))
    wt = w[0] if cut is None else w
    y, _ = R.rft_linear(x, wt, groups=groups)
    dx, dw, db = R.rft_linear_bwd(dy, x, wt, groups=groups, dw_dtype=F32, want_db=True)
    dw, db = dw.view(E, n, k), db.view(E, n)
    # fp32 products of whole numbers are exact in any order while no sum passes 2^24
    for e, (a, b) in enumerate(((0, rows),) if cut is None else ((0, cut), (cut, rows))):
        sum_w, sum_b = torch.zeros(n, k, device=DEV), torch.zeros(n, device=DEV)
        for i in range(a, b, 100_000):
            j = min(b, i + 100_000)
            xf, df, wf = x[i:j].float(), dy[i:j].float(), w[e].float()
            assert torch.equal(y[i:j], (xf @ wf.t().contiguous()).to(dt)), (e, i)
            assert torch.equal(dx[i:j], (df @ wf).to(dt)), (e, i)
            sum_w += df.t().contiguous() @ xf
            sum_b += df.sum(0)
        assert torch.equal(dw[e], sum_w) and torch.equal(db[e], sum_b)


@pytest.mark.parametrize("count", (5, 700))
def test_sources_at_the_end_of_the_largest_array(count):
    """bf16: byte offsets of a source's rows up to 2^32."""
    k, n = 2048, 32
    tokens = ((1 << 31) - 64) // k
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.zeros(tokens, k, dtype=BF, device=DEV)
    x[-64:], x[:64] = whole(g, 64, k, BF), whole(g, 64, k, BF)
    near = torch.randint(0, 64, (count,), generator=g, device=DEV)
    source = torch.where(torch.arange(count, device=DEV) % 3 > 0, tokens - 1 - near, near).int()
    source[0], source[-1] = tokens - 1, tokens  # the last row, and one behind it
    w, dy = whole(g, n, k, BF), whole(g, count, n, BF)
    rows = torch.cat([x[source[:-1].long()], torch.zeros(1, k, dtype=BF, device=DEV)]).float()
    groups = R.Groups(None, source)
    y, _ = R.rft_linear(x, w, groups=groups)
    assert torch.equal(y, (rows @ w.float().t().contiguous()).to(BF))
    dx, dw, _ = R.rft_linear_bwd(dy, x, w, groups=groups, dw_dtype=F32)
    assert torch.equal(dx, (dy.float() @ w.float()).to(BF))
    assert torch.equal(dw, dy.float().t().contiguous() @ rows)

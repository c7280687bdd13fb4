"""d_weight in fp32 from bf16 data behind an activation: the products take dz in two bf16 parts, so
that an fp32 result is not that of dz rounded to bf16; one product where the caller asks for it.

Tolerances.  dz is off by 2^-19 of its terms (the activation's slope, as in the other tests of these
layers); its first part by half a step, 2^-8 of dz, its second by 2^-8 of what that left: 2^-16.
Products are exact in fp32, sums of K terms within (K + 3) 2^-23 of their magnitudes, for each of the
two products, and their sum is rounded once more."""
import math

import pytest
import torch

import paper_2505_17826_amd as R
from tests import linear_model as M
from tests.gpu_cases import requires_gpu
from tests.test_linear_gpu import Case, CODE

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")
BF, F32 = torch.bfloat16, torch.float32


def want(c, z):
    """d_weight in 64 bits, the error that dz may have, and the sums of magnitudes."""
    _, rw, _, dz, _, mw, _ = M.backward(c.dy.double(), z.double(), c.xr, c.w.double(), c.act, c.offsets)
    zz = z.double()[:c.live]
    gate = zz[:, :c.m] if c.act == "swiglu" else zz
    amp = c.dy.double()[:c.live].abs() * (1 + gate.abs())
    if c.act == "swiglu":
        amp = torch.cat([amp * zz[:, c.m:].abs(), amp], 1)
    amp, dz, x = amp * 2.0 ** -19, dz[:c.live].abs(), c.xr[:c.live].abs()

    def products(a):
        out = torch.zeros_like(rw)
        for e in range(c.E):
            i, j = c.offsets[e], c.offsets[e + 1]
            out[e] = a[i:j].T @ x[i:j]
        return out

    return rw, products(amp), products(dz), mw


def tolerances(c, z):
    rw, amp, mag, mw = want(c, z)
    most = max(b - a for a, b in zip(c.offsets, c.offsets[1:]))
    acc = (most + 3) * 2.0 ** -23 * 1.01  # 1.01: the magnitudes with their own errors
    two = amp + 2.0 ** -16 * (mag + amp) + 2 * acc * mw
    one = amp + 2.0 ** -8 * (mag + amp) + acc * mw
    return rw, two, one


def run(c, z, **kw):
    d = c.dev
    return R.rft_linear_bwd(d(c.dy), d(c.x), d(c.w), z=d(z), act=CODE[c.act], groups=c.groups(),
                            dw_dtype=F32, want_dx=False, **kw)[1].cpu().double()


def z_of(c):
    return torch.randn(c.rows, c.n, generator=torch.Generator().manual_seed(5)).to(c.dt)


CASES = [([37, 0, 140], 72, 208, 3), ([5000], 40, 64, 0), ([700, 0, 1, 2085, 3], 328, 4176, 2), ([1], 8, 16, 0)]


@pytest.mark.parametrize("act", ("silu", "gelu", "swiglu"))
@pytest.mark.parametrize("counts,k,n,spare", CASES)
def test_fp32_d_weight(counts, k, n, spare, act):
    c = Case(counts, k, n, act, BF, spare=spare, seed=k)
    z = z_of(c)
    rw, two, one = tolerances(c, z)
    got = run(c, z)
    assert bool(((got - rw).abs() <= two + 2.0 ** -24 * (rw.abs() + two) + 1e-30).all()), \
        float(((got - rw).abs() / (two + 1e-30)).max())
    dw0 = torch.randn(c.w.shape, generator=torch.Generator().manual_seed(9))
    got = run(c, z, d_weight=dw0.to(DEV), accumulate=True)
    t = two + 2.0 ** -23 * (rw.abs() + two + dw0.double().abs())  # two sums of it
    assert bool(((got - rw - dw0.double()).abs() <= t + 1e-30).all())
    fast = run(c, z, one_product=True)
    assert bool(((fast - rw).abs() <= one + 2.0 ** -24 * (rw.abs() + one) + 1e-30).all())
    if sum(counts) > 1000:
        off = lambda a: float((a - rw).norm() / rw.norm())  # noqa: E731
        # 2^-16 at most, against about 2^-9 of values rounded at random
        assert off(run(c, z)) < 2.0 ** -16 < 2.0 ** -11 < off(fast)


@pytest.mark.parametrize("act", ("silu", "swiglu"))
def test_d_weight_of_a_dense_layer_with_cut_tiles(act):
    """272 tiles of 256 x 256, the last ones cut along the rows, against 64 bits on the GPU."""
    rows, k, n = 2100, 4096, 4352
    g = torch.Generator(device=DEV).manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    m = n // 2 if act == "swiglu" else n
    x, w, dy, z = r(rows, k).to(BF), (r(n, k) / 64).to(BF), r(rows, m).to(BF), r(rows, n).to(BF)
    got = R.rft_linear_bwd(dy, x, w, z=z, act=CODE[act], dw_dtype=F32, want_dx=False)[1].double()
    dz = torch.cat([dy.double() * s for s in M.slopes(z.double(), act)], 1).T.contiguous()
    rw = dz @ x.double()
    # 2100 terms rounded by 2^-16 of each at random, the sums by 2^-23 of theirs
    assert float((got - rw).norm() / rw.norm()) < 2.0 ** -16


def test_results_of_other_types_are_those_of_one_product():
    """d_weight in bf16, or without an activation, and d_x and d_bias with either."""
    c = Case([300, 7], 136, 160, "swiglu", BF, seed=2)
    z, d = z_of(c), c.dev
    call = lambda **kw: R.rft_linear_bwd(d(c.dy), d(c.x), d(c.w), z=d(z), act=CODE[c.act],  # noqa: E731
                                         groups=c.groups(), want_db=True, **kw)
    a, b, e = call(), call(dw_dtype=F32), call(dw_dtype=F32, one_product=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])
    assert torch.equal(a[0], e[0]) and torch.equal(a[2], e[2])
    assert torch.equal(a[1], e[1].to(BF)) and not torch.equal(b[1], e[1])
    c = Case([300, 7], 136, 160, "none", BF, seed=2)
    a, b = (R.rft_linear_bwd(d(c.dy), d(c.x), d(c.w), groups=c.groups(), dw_dtype=F32, one_product=p)[1]
            for p in (False, True))
    assert torch.equal(a, b)


def test_values_without_a_second_part():
    """A dz that is infinite, NaN or past bf16 has no second part, and only its own columns show it."""
    n, k = 16, 8
    dy = torch.ones(4, n).to(BF)
    z = torch.full((4, n), 30.0).to(BF)  # slope of silu 1
    dy[0, 3], dy[1, 5] = math.inf, math.nan
    x = torch.ones(4, k).to(BF)
    w = torch.zeros(n, k).to(BF)
    dw = R.rft_linear_bwd(dy.to(DEV), x.to(DEV), w.to(DEV), z=z.to(DEV), act=R.RFT_ACT_SILU, dw_dtype=F32,
                          want_dx=False)[1].cpu()
    assert bool((dw[3] == math.inf).all()) and bool(dw[5].isnan().all())
    fine = [i for i in range(n) if i not in (3, 5)]
    assert bool((dw[fine] == 4).all())


def test_two_parts_in_a_replayed_graph():
    c = Case([100, 0, 31, 400], 136, 96, "gelu", BF, seed=6)
    d, z = c.dev, z_of(c)
    x, w, dy, zd, groups = d(c.x), d(c.w), d(c.dy), d(z), c.groups()
    call = lambda: R.rft_linear_bwd(dy, x, w, z=zd, act=CODE[c.act], groups=groups, dw_dtype=F32)[:2]  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for i in range(3):
        x.mul_(-1.25)
        for t in held:
            t.zero_()
        graph.replay()
        again = call()
        torch.cuda.synchronize()
        assert torch.equal(held[0], again[0]) and torch.equal(held[1], again[1]), i

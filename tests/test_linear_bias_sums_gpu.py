"""d_bias of long and of crowded groups: at most 128 additions to a running fp32 sum, joined in fp64.

With every dz the same a running sum rounds the same way at each step, so its error does not
average out: 2^-24 of the sum for each addition.  128 additions are 2^-17 of the sum at most, the
join of them is exact to 2^-50, and the result is rounded once, 2^-24."""
import pytest
import torch

import paper_2505_17826_amd as R
from tests.gpu_cases import requires_gpu

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")
TOL = 2.0 ** -17 + 2.0 ** -23


def d_bias(dy, offsets, E, n, **kw):
    x, w = torch.zeros(dy.shape[0], 8, dtype=dy.dtype, device=DEV), torch.zeros(E, n, 8, dtype=dy.dtype, device=DEV)
    g = R.Groups(torch.tensor(offsets, dtype=torch.int32, device=DEV))
    return R.rft_linear_bwd(dy, x, w, groups=g, want_dx=False, want_dw=False, want_db=True, **kw)[2]


@pytest.mark.parametrize("n", (16, 17))
@pytest.mark.parametrize("E", (1, 1024))
def test_equal_terms(E, n):
    rows = 1 << 21
    at = E // 2
    dy = torch.full((rows, n), 1 / 3, device=DEV)
    db = d_bias(dy, [0] * (at + 1) + [rows] * (E - at), E, n).double()
    want = float(dy[0, 0].double()) * rows
    assert bool(((db[at] - want).abs() <= TOL * want).all()), float((db[at] - want).abs().max() / want)
    db[at] = 0
    assert not db.any()


def test_equal_terms_bf16_behind_an_activation():
    """swiglu: both halves."""
    rows, E, m = 1 << 20, 512, 8
    dy = torch.full((rows, m), 0.33203125, device=DEV).to(torch.bfloat16)
    z = torch.cat([torch.full((rows, m), 0.7), torch.full((rows, m), 0.9)], 1).to(torch.bfloat16).to(DEV)
    db = d_bias(dy, [0] + [rows] * E, E, 2 * m, z=z, act=R.RFT_ACT_SWIGLU).double()[0]
    g, u, d = (float(t) for t in (z[0, 0].double(), z[0, m].double(), dy[0, 0].double()))
    s = torch.sigmoid(torch.tensor(g, dtype=torch.float64)).item()
    for got, term in ((db[:m], d * u * s * (1 + g * (1 - s))), (db[m:], d * g * s)):
        # the term itself: 2^-19, as in the other tests of these activations
        assert bool(((got / (term * rows) - 1).abs() <= TOL + 2.0 ** -19).all()), got


def test_terms_of_both_signs():
    rows, E, n = 300_001, 64, 24
    g = torch.Generator(device=DEV).manual_seed(1)
    dy = torch.randn(rows, n, generator=g, device=DEV)
    off = [0, 1, rows - 130] + [rows] * (E - 2)
    db = d_bias(dy, off, E, n).double()
    for e in range(3):
        a, b = off[e], off[e + 1]
        want, mag = dy[a:b].double().sum(0), dy[a:b].double().abs().sum(0)
        assert bool(((db[e] - want).abs() <= 2.0 ** -17 * mag + 2.0 ** -24 * want.abs()).all())

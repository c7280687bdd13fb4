"""d_bias on bf16 data is summed from dz as it is before its rounding for the products.

Tolerance: dz is off by 2^-19 of its terms (the activation's slope), 128 of a lane's rows are summed in
fp32, (128 + 8) 2^-24 of their magnitudes, and the result is rounded once, 2^-24.  Nothing in it is of
the size of a rounding of dz to bf16; that a sum of rounded terms is refused is tested on the CPU."""
import pytest
import torch

from tests import linear_model as M
from tests.gpu_cases import requires_gpu
from tests.test_linear_gpu import Case, CODE

import paper_2505_17826_amd as R

pytestmark = [pytest.mark.gpu, requires_gpu]
BF = torch.bfloat16
ACTS = ("silu", "gelu", "swiglu")
COUNTS = [([37, 0, 140], 208), ([5000], 64), ([1, 300, 2], 80)]


def make(counts, n, act):
    c = Case(counts, 16, n, act, BF, seed=n)
    return c, torch.randn(c.rows, n, generator=torch.Generator().manual_seed(5)).to(BF)


def want(c, z):
    """d_bias in 64 bits and what it may be off."""
    _, _, rb, dz, _, _, mb = M.backward(c.dy.double(), z.double(), c.xr, c.w.double(), c.act, c.offsets)
    zz = z.double()
    gate = zz[:, :c.m] if c.act == "swiglu" else zz
    amp = c.dy.double().abs() * (1 + gate.abs())
    if c.act == "swiglu":
        amp = torch.cat([amp * zz[:, c.m:].abs(), amp], 1)
    amp = torch.stack([amp[a:b].sum(0) for a, b in zip(c.offsets, c.offsets[1:])]) * 2.0 ** -19
    return rb, amp + 136 * 2.0 ** -24 * (mb + amp) + 2.0 ** -24 * rb.abs() + 1e-30, dz


@pytest.mark.parametrize("products", (False, True))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("counts,n", COUNTS)
def test_sums_of_unrounded_terms(counts, n, act, products):
    """Alone, and beside the products."""
    c, z = make(counts, n, act)
    d = c.dev
    db = R.rft_linear_bwd(d(c.dy), d(c.x), d(c.w), z=d(z), act=CODE[act], groups=c.groups(), want_dx=products,
                          want_dw=products, want_db=True)[2].cpu().double()
    rb, tol, _ = want(c, z)
    assert bool(((db - rb).abs() <= tol).all()), float(((db - rb).abs() / tol).max())

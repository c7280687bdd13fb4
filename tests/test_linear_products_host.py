"""What the GPU tests of d_weight in fp32 rest on (no GPU needed): their tolerances refuse a dz that
is rounded to bf16 once, and the library refuses the flag with other types."""
import ctypes

import pytest
import torch

import paper_2505_17826_amd as R
from tests import linear_model as M
from tests.test_linear_products_gpu import BF, CASES, Case, tolerances, z_of


def products(c, dz):
    out = torch.zeros(c.w.shape, dtype=torch.float64)
    for e in range(c.E):
        i, j = c.offsets[e], c.offsets[e + 1]
        out[e] = dz[i:j].T @ c.xr[i:j]
    return out


@pytest.mark.parametrize("act", ("silu", "gelu", "swiglu"))
def test_tolerances_tell_one_part_from_two(act):
    counts, k, n, spare = CASES[0]
    c = Case(counts, k, n, act, BF, spare=spare, seed=k)
    z = z_of(c)
    dz = torch.cat([c.dy.double() * s for s in M.slopes(z.double(), act)], 1)
    rw, two, one = tolerances(c, z)
    first = dz.to(BF).double()
    second = (dz - first).to(BF).double()
    a, b = (products(c, first) - rw).abs(), (products(c, first + second) - rw).abs()
    assert bool((b <= two + 1e-30).all()) and bool((a <= one + 1e-30).all())
    assert not bool((a <= two).all())


def test_flag_of_one_product():
    L, fake = R.lib(), ctypes.c_void_p(0x1000)

    def status(dt, dwt):  # no workspace: nothing is enqueued
        g = ctypes.byref(R.rft_groups(16, 2, 0x1000, None, 1, 0))
        return L.rft_linear_bwd(g, fake, fake, fake, fake, dt, 64, 32, R.RFT_ACT_SILU, fake, fake, dwt, fake, 1,
                                None, 0, None)

    assert status(R.RFT_BF16, R.RFT_F32 | R.RFT_ONE_PRODUCT) == R.RFT_E_WORKSPACE
    assert status(R.RFT_F32, R.RFT_F32 | R.RFT_ONE_PRODUCT) == R.RFT_E_WORKSPACE
    for dt in (R.RFT_BF16, R.RFT_F32):
        assert status(dt, R.RFT_BF16 | R.RFT_ONE_PRODUCT) == R.RFT_E_DTYPE
        assert status(dt, 2 * R.RFT_ONE_PRODUCT) == R.RFT_E_DTYPE

"""The tolerance of the GPU test of d_bias refuses a sum of dz rounded to bf16 (no GPU needed)."""
import pytest
import torch

from tests.test_linear_bias_gpu import ACTS, BF, COUNTS, make, want


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("counts,n", COUNTS)
def test_sums_of_rounded_terms_are_refused(counts, n, act):
    c, z = make(counts, n, act)
    rb, tol, dz = want(c, z)
    sums = lambda t: torch.stack([t[a:b].sum(0) for a, b in zip(c.offsets, c.offsets[1:])])  # noqa: E731
    assert bool(((sums(dz) - rb).abs() <= tol).all())
    assert not bool(((sums(dz.to(BF).double()) - rb).abs() <= tol).all())

"""Few rows per group on average and most of them in one: every row by its own group's weight, in groups
of any number of passes, exactly (whole numbers, sums below 2^24)."""
import pytest
import torch

import paper_2505_17826_amd as R
from tests.gpu_cases import requires_gpu

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")
BF = torch.bfloat16


def crowd(E, rows, at, others=0):
    c = [others] * E
    c[at] += rows
    return c


COUNTS = [crowd(1024, 4000, 700), crowd(1024, 2100, 0, 1), crowd(64, 1601, 63), crowd(5, 70, 2, 3),
          [0] * 255 + [65] + [0] * 3 + [129, 1, 0, 64] + [0] * 250, [16, 17, 0, 31, 33] * 60, crowd(300, 0, 5, 1),
          [128, 0, 0, 0, 0, 0, 1], [0] * 7]


@pytest.mark.parametrize("act", ("none", "swiglu"))
@pytest.mark.parametrize("i", range(len(COUNTS)))
def test_whole_numbers(i, act):
    counts = COUNTS[i]
    E, k, n, live = len(counts), 264, 208, sum(counts)
    spare = 3
    g = torch.Generator(device=DEV).manual_seed(i)
    whole = lambda *s: torch.randint(-2, 3, s, generator=g, device=DEV).to(BF)  # noqa: E731
    source = torch.randint(0, 50 * 3, (live + spare,), generator=g, device=DEV, dtype=torch.int32)
    x, w, res = whole(50, k), whole(E, n, k), whole(live + spare, n)
    offsets = torch.tensor([0] + counts).cumsum(0)
    groups = R.Groups(offsets.int().to(DEV), source, 3)
    expert = torch.repeat_interleave(torch.arange(E), torch.tensor(counts)).to(DEV)
    rows = x[(source[:live] // 3).long()].float()
    z = torch.cat([(w[expert[a:a + 500]].float() * rows[a:a + 500, None, :]).sum(2) for a in range(0, live, 500)]
                  or [torch.zeros(0, n, device=DEV)])
    if act == "none":
        out = torch.full((live + spare, n), 7.0, dtype=BF, device=DEV)
        y, _ = R.rft_linear(x, w, residual=res, groups=groups, out=out)
        assert torch.equal(y[:live], (z + res[:live].float()).to(BF)) and bool((y[live:] == 7).all())
        return
    kept = torch.full((live + spare, n), 7.0, dtype=BF, device=DEV)
    y, kept = R.rft_linear(x, w, act=R.RFT_ACT_SWIGLU, groups=groups, z=kept)
    assert torch.equal(kept[:live], z.to(BF)) and bool((kept[live:] == 7).all())
    h = n // 2
    want = z[:, :h].double() * torch.sigmoid(z[:, :h].double()) * z[:, h:].double()
    # the sigmoid 2^-19 of its value where it is below fp32's range nothing; one rounding
    tol = (2.0 ** -8 + 2.0 ** -18) * want.abs() + 2.0 ** -100
    assert bool(((y[:live].double() - want).abs() <= tol).all())


def test_slices_and_crowds():
    """Few blocks: the summed index in slices, more passes than groups."""
    counts = [0, 100, 1, 0, 19]
    k, n, live = 4104, 48, 120
    g = torch.Generator(device=DEV).manual_seed(1)
    whole = lambda *s: torch.randint(-2, 3, s, generator=g, device=DEV).to(BF)  # noqa: E731
    x, w = whole(live, k), whole(5, n, k)
    groups = R.Groups(torch.tensor([0] + counts).cumsum(0).int().to(DEV))
    y, _ = R.rft_linear(x, w, groups=groups)
    a = 0
    for e, c in enumerate(counts):
        assert torch.equal(y[a:a + c], (x[a:a + c].float() @ w[e].float().t().contiguous()).to(BF))
        a += c


def test_offsets_that_are_not_valid_stay_inside():
    """Passes beyond the rows: values are unspecified, places only those of the rows."""
    x, w = torch.randn(300, 64, device=DEV).to(BF), torch.randn(40, 64, 64, device=DEV).to(BF)
    for off in ([300 if i % 2 else 0 for i in range(41)], [2 ** 31 - 1 if i % 3 else -5 for i in range(41)]):
        buf = torch.full((302 * 64,), 7.0, dtype=BF, device=DEV)
        R.rft_linear(x, w, groups=R.Groups(torch.tensor(off, dtype=torch.int32, device=DEV)),
                     out=buf[64:301 * 64].view(300, 64))
        assert (buf[:64] == 7).all() and (buf[301 * 64:] == 7).all()

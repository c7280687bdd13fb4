"""Weight decay at fine-tuning rates.  lr * weight_decay of 1e-8 to 1e-7 is less than fp32 can
tell 1 - lr * weight_decay from 1, but not less than it moves a weight together with its
step; the mean over many weights, whose roundings are as often up as down, shows it."""
import math

import pytest
import torch

import paper_2505_17826_amd as R
from tests.gpu_cases import requires_gpu

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")

RATES = [(1e-6, 0.01), (1e-6, 0.1), (1e-5, 0.01), (3e-6, 0.013)]


def limit(n, decay):
    """The mean rounding of n results in [1, 2), each uniform within 2^-24 (half a step): six
    standard deviations; and the decay's own factors, 2^-23 of it."""
    return 6 * 2.0 ** -24 / math.sqrt(3 * n) + 2.0 ** -23 * decay


@pytest.mark.parametrize("lr,wd", RATES)
@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("offset", [0, 1])
def test_adamw(lr, wd, master, offset):
    n = 1 << 20
    g = torch.Generator(DEV).manual_seed(7)
    buf = torch.rand(n + offset, generator=g, device=DEV)
    w = (1.0 + 2.0 ** -10 + buf * (1 - 2.0 ** -9))[offset:]
    m = torch.randn(n, generator=g, device=DEV)
    v = 0.5 + torch.rand(n, generator=g, device=DEV)
    grad = torch.zeros(n, device=DEV)
    w0, m0, v0 = w.double(), m.double(), v.double()
    low = w.to(torch.bfloat16)
    b1, b2, eps, step = 0.9, 0.95, 1e-8, 30
    t = (low, grad, m, v, w) if master else (w, grad, m, v)
    R.rft_adamw_step(R.Params([t]), R.adamw_params(lr, b1, b2, eps, wd, step))
    hat = (b2 * v0 / (1 - b2 ** step)).sqrt() + eps
    s = lr * (b1 * m0 / (1 - b1 ** step)) / hat
    # the step's own rounding is some 2^-24 of 1e-5 for each weight
    decay = float((w0 - s - w.double()).mean())
    want = lr * wd * float(w0.mean())
    assert abs(decay - want) <= limit(n, want) + 16 * 2.0 ** -24 * float(s.abs().mean()), (decay, want)
    if master:
        assert torch.equal(low, w.to(torch.bfloat16))


@pytest.mark.parametrize("lr,wd", RATES)
@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("shape", [(100, 8192), (8192, 99), (1024, 1024), (1023, 1025), (4, 400, 700),
                                   (40, 300, 264)])
def test_muon_step(lr, wd, master, shape):
    n = math.prod(shape)
    g = torch.Generator(DEV).manual_seed(9)
    rows, cols = shape[-2:]
    w = 1.0 + 2.0 ** -10 + torch.rand(shape, generator=g, device=DEV) * (1 - 2.0 ** -9)
    u = torch.randn(shape, generator=g, device=DEV)
    w0 = w.double()
    low = w.to(torch.bfloat16)
    scale = math.sqrt(max(rows, cols))  # entries of the update of lr in size: many fp32 steps
    prm = lambda **kw: R.muon_params(products=R.RFT_PRODUCTS_THREE, **kw)  # noqa: E731
    R.rft_muon_step(low if master else w, u, None, prm(lr=lr, weight_decay=wd, scale=scale),
                    master=w if master else None)
    s = lr * scale * R.rft_orthogonalize(u, prm()).double()
    decay = float((w0 - s - w.double()).mean())
    want = lr * wd * float(w0.mean())
    assert abs(decay - want) <= limit(n, want) + 4 * 2.0 ** -24 * float(s.abs().mean()), (decay, want)
    if master:
        assert torch.equal(low, w.to(torch.bfloat16))

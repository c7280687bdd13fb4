"""rft_orthogonalize and rft_muon_step within the documented errors, on every tile size in both
orientations: single matrices and stacks whose products take tiles of 64, 128 (two depths) and
256 rows, results and weights of every type, a matrix alone and in its stack."""
import pytest
import torch

import paper_2505_17826_amd as R
from tests import ortho_model as M
from tests.gpu_cases import requires_gpu
from tests.test_ortho_model_host import SHAPES

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")
f32, bf16 = torch.float32, torch.bfloat16
# products with X of 4 x 6 tiles a matrix: 48 tiles in all (64 rows), 144 and 480 (128), 960 (256)
STACKS = [2, 6, 20, 40]


@pytest.mark.parametrize("shape", SHAPES + [(100, 4000), (1000, 1100), (2300, 1100), (3, 9000), (9000, 3)])
def test_documented_errors(shape):
    g = M.gradient(shape[0] * 31 + shape[1], *shape)
    x = g.to(DEV)
    o = R.rft_orthogonalize(x, R.muon_params(products=R.RFT_PRODUCTS_ONE)).cpu()
    assert M.error(o, g) <= M.ONE, M.error(o, g)
    o = R.rft_orthogonalize(x, R.muon_params(products=R.RFT_PRODUCTS_THREE)).cpu()
    assert M.error(o, g) <= M.three(g), (M.error(o, g), M.three(g))


@pytest.mark.parametrize("tall", [True, False])
@pytest.mark.parametrize("batch", STACKS)
def test_stacks_of_every_tile_size(batch, tall):
    shape = (batch, 768, 512) if tall else (batch, 512, 768)
    g = M.gradient(batch, *shape)
    x = g.to(DEV)
    some = sorted({0, batch // 2, batch - 1})
    for products, limit in ((R.RFT_PRODUCTS_ONE, M.ONE), (R.RFT_PRODUCTS_THREE, M.three(g[some]))):
        p = R.muon_params(products=products)
        o = R.rft_orthogonalize(x, p)
        assert M.error(o[some].cpu(), g[some]) <= limit
        assert torch.equal(R.rft_orthogonalize(x, p, out_dtype=bf16), o.to(bf16))
        for i in some:
            assert torch.equal(R.rft_orthogonalize(x[i], p), o[i])


@pytest.mark.parametrize("tall", [True, False])
@pytest.mark.parametrize("batch", STACKS + [1])
@pytest.mark.parametrize("wdt,master", [(f32, False), (bf16, True), (bf16, False)])
def test_steps_of_every_tile_size(batch, tall, wdt, master):
    lr, mu, wd, scale = 0.05, 0.9, 0.1, 1.5
    # one matrix of more than 128 tiles, or a stack
    m, n = (768, 512) if batch > 1 else (2300, 1100)
    shape = (batch, m, n) if tall else (batch, n, m)
    g, buf, w0 = (M.gradient(s + batch, *shape) for s in (1, 2, 3))
    prm = R.muon_params(lr, mu, True, wd, scale)
    some = sorted({0, batch // 2, batch - 1})
    gd, bd, wd0 = g.to(DEV), buf.to(DEV), w0.to(DEV)
    ms = wd0.clone() if master else None
    w, b1 = wd0.to(wdt), bd.clone()
    start = w.clone()
    R.rft_muon_step(w, gd, b1, prm, master=ms)
    u = [(mu * (mu * buf[i].double() + (1 - mu) * g[i].double()) + (1 - mu) * g[i].double()) for i in some]
    got = w if ms is None else ms
    one = got.dtype == bf16
    for i, ui in zip(some, u):
        base = (wd0 if master else start)[i].double().cpu()
        step = lr * scale * M.iterate(ui)
        d = got[i].double().cpu() - (base * (1 - lr * wd) - step)
        # the update's error, and the roundings of the weight (bf16: 2^-8 at most; fp32: of the
        # momentum and of the change, three)
        limit = (M.ONE if one else M.three(ui.float())) * float(step.norm())
        limit += (2.0 ** -8 if one else 3 * 2.0 ** -24) * float(base.norm() + step.norm())
        assert float(d.norm()) <= limit
        # the same bits as the matrix alone
        w1, b2 = start[i].clone(), bd[i].clone()
        m1 = wd0[i].clone() if master else None
        R.rft_muon_step(w1, gd[i], b2, prm, master=m1)
        assert torch.equal(w1, w[i]) and torch.equal(b2, b1[i])
        assert m1 is None or torch.equal(m1, ms[i])
    if master:
        assert torch.equal(w, ms.to(wdt))

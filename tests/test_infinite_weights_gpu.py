"""Weights that are not finite (places masked with -inf) under AdamW and the momentum step: an
infinite weight keeps its value, with decay and without, a NaN stays NaN, and neither touches
its neighbours."""
import math

import pytest
import torch

import paper_2505_17826_amd as R
from tests.gpu_cases import requires_gpu

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")
BAD = (math.inf, -math.inf, math.nan)


def planted(shape, seed, dtype):
    g = torch.Generator(DEV).manual_seed(seed)
    w = torch.randn(shape, generator=g, device=DEV)
    bad = w.clone()
    bad.view(-1)[7:16] = torch.tensor(3 * BAD, device=DEV)
    return w.to(dtype), bad.to(dtype)


def same(got, want, bad):
    at = ~torch.isfinite(bad)
    assert torch.equal(got[~at], want[~at])
    # a master is compared with the bf16 weight of the same infinities
    assert torch.equal(got[at].float().nan_to_num(0.5), bad[at].float().nan_to_num(0.5))


@pytest.mark.parametrize("wd", [0.0, 0.1])
@pytest.mark.parametrize("dtype,master", [(torch.float32, False), (torch.bfloat16, False),
                                          (torch.bfloat16, True)])
@pytest.mark.parametrize("n", [1000, 1003])
def test_adamw(wd, dtype, master, n):
    grad = torch.randn(n, device=DEV)
    res = []
    for w in planted(n, 1, dtype):
        ms = w.float() if master else None
        m, v = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
        R.rft_adamw_step(R.Params([(w, grad, m, v, ms)]), R.adamw_params(1e-3, weight_decay=wd))
        res.append((w, ms))
    bad = planted(n, 1, dtype)[1]
    same(res[1][0], res[0][0], bad)
    if master:
        same(res[1][1], res[0][1], bad)


@pytest.mark.parametrize("wd", [0.0, 0.1])
@pytest.mark.parametrize("dtype,master", [(torch.float32, False), (torch.bfloat16, False),
                                          (torch.bfloat16, True)])
@pytest.mark.parametrize("shape", [(40, 64), (41, 63), (200, 304), (301, 155)])
def test_muon_step(wd, dtype, master, shape):
    grad = torch.randn(shape, device=DEV)
    res = []
    for w in planted(shape, 2, dtype):
        ms = w.float() if master else None
        R.rft_muon_step(w, grad, None, R.muon_params(weight_decay=wd), master=ms)
        res.append((w, ms))
    bad = planted(shape, 2, dtype)[1]
    same(res[1][0], res[0][0], bad)
    if master:
        same(res[1][1], res[0][1], bad)

"""The router on rows whose largest logit is far from 0 (every expert filled with -1e9 or
-1e30, a drifted router): the softmax depends on the differences alone, so p, the gates, the
selection and the gradient of such a row are as accurate as those of a row near 0, and the
losses of the rows beside it stay finite."""
import math

import numpy as np
import pytest
import torch

import paper_2505_17826_amd as R
from tests.gpu_cases import requires_gpu
from tests.test_router_gpu import reference

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")


def rows(E, dtype, seed, huge):
    """Ordinary rows, rows about a large level (their differences kept by the type or not), and
    filled ones; float64 as the device holds them, and the device's."""
    g = torch.Generator().manual_seed(seed)
    noise = lambda: 2.0 * torch.randn(E, generator=g)  # noqa: E731
    fill = lambda x: torch.full((E,), x)  # noqa: E731
    z = [noise(), noise() - 65504.0, noise() + 1000.0, fill(-1e9), noise(), fill(1e9),
         64.0 * noise() - 1e9, fill(-65504.0), 1e4 * noise()]
    if huge:
        z += [fill(-1e30), fill(1e10), noise(), fill(3e37), fill(-1.9e38), 1e30 * noise(),
              torch.cat([fill(-1e30)[:E // 2], fill(-math.inf)[E // 2:]])]
    z = torch.stack(z).to(dtype)
    return z.double().numpy(), z.to(DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E,k", [(8, 2), (20, 3), (60, 4), (128, 8), (250, 8), (300, 5), (1024, 16)])
@pytest.mark.parametrize("huge", [False, True])
def test_large_logits(E, k, dtype, huge):
    zr, zd = rows(E, dtype, E + k, huge)
    T = zd.shape[0]
    starts, mask = [0, 3, 5, T], [1] * T
    # the z-loss of rows of 1e30 is past fp32
    cb, cz = 0.5, 0.0 if huge else 1e-12
    tok = R.Tokens(torch.tensor(starts, dtype=torch.int32, device=DEV),
                   torch.tensor(mask, dtype=torch.uint8, device=DEV))
    dg = torch.randn(T, k, generator=torch.Generator().manual_seed(E))
    # a value's error relative to itself: its exponent |x - max| (at most 104 ln 2 where the value is
    # not 0) rounded twice, the exponential, E sums and a division by a few 2^-24
    tol = (2 * 104 * math.log(2) + 8 + math.log2(E) + 4) * 2.0 ** -24
    for norm in (True, False):
        for scope in (R.RFT_BALANCE_BATCH, R.RFT_BALANCE_ROLLOUT):
            prm = R.router_params(E, k, norm_topk=norm, balance_coef=cb, z_coef=cz, scope=scope)
            ref = reference(zr, mask, starts, E, k, norm, scope == R.RFT_BALANCE_ROLLOUT, cb, cz,
                            dg.double().numpy())
            o = R.rft_router_fwd(tok, zd, prm)
            st = R.stats_to_dict(o.stats, R.rft_router_stats)
            assert np.array_equal(o.expert_ids.cpu().numpy(), ref["ids"])
            assert np.array_equal(o.counts.cpu().numpy(), ref["counts"])
            gates = o.gates.cpu().double().numpy()
            assert np.all(np.abs(gates - ref["gates"]) <= 2 * tol * ref["gates"] + 1e-37)
            assert np.all(np.abs(o.lse.cpu().double().numpy() - ref["lse"]) <=
                          2 * tol + 2.0 ** -23 * np.abs(ref["lse"]))
            assert abs(st["balance_loss"] - ref["bal"]) <= 4 * tol * ref["bal"]
            if not huge:
                assert abs(st["z_loss"] - ref["zl"]) <= 2.0 ** -21 * ref["zl"]
                assert abs(st["loss"] - ref["loss"]) <= 4 * tol * ref["loss"]
            else:
                assert abs(st["loss"] - ref["loss"]) <= 4 * tol * ref["loss"]
            d = R.rft_router_bwd(tok, zd, prm, o, d_gates=dg.to(DEV)).cpu().double().numpy()
            half = torch.finfo(dtype).eps / 2
            # as for ordinary rows: p and dp each carry tol, twice more in the normed gates
            lim = 8 * tol * (1 + E ** 0.5 / 8) * ref["scale"] + half * np.abs(ref["dz"]) + 1e-36
            worst = (np.abs(d - ref["dz"]) / lim).max(1)
            assert np.all(worst <= 1), worst
            s = R.rft_router_fwd(tok, zd, prm, want_loss=False)
            assert torch.equal(s.expert_ids, o.expert_ids) and torch.equal(s.gates, o.gates)

"""The router over many rows where a whole wave works on a row (more than 256 experts) and with
bf16 logits, forward and backward with the gates' gradients, against torch in float64 on the
device."""
import numpy as np
import pytest
import torch

import paper_2505_17826_amd as R
from tests.gpu_cases import requires_gpu

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E,k", [(96, 8), (200, 6), (300, 8), (512, 8), (1000, 16)])
@pytest.mark.parametrize("scope", [R.RFT_BALANCE_BATCH, R.RFT_BALANCE_ROLLOUT])
def test_many_rows(E, k, dtype, scope):
    r = np.random.default_rng(E + k)
    lens = r.integers(0, 1500, 40).tolist() + [0, 1, 2]
    T, S0 = int(sum(lens)), len(lens)
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    g = torch.Generator(DEV).manual_seed(E)
    z = (2 * torch.randn((T, E), device=DEV, generator=g)).to(dtype)
    dg = torch.randn((T, k), device=DEV, generator=g)
    mask = torch.from_numpy((r.random(T) < 0.9).astype(np.uint8)).to(DEV)
    tok = R.Tokens(torch.from_numpy(starts).to(DEV), mask)
    cb, cz = 0.5, 0.01
    m = mask.bool()
    zd = z.double()
    lse = torch.logsumexp(zd, 1) * m
    p = torch.softmax(zd, 1) * m[:, None]
    ids = torch.argsort(z.float(), dim=1, descending=True, stable=True)[:, :k]
    hot = torch.zeros((T, E), dtype=torch.float64, device=DEV).scatter_(1, ids, 1.0) * m[:, None]
    by = scope == R.RFT_BALANCE_ROLLOUT
    G = S0 if by else 1
    sg = torch.repeat_interleave(torch.arange(S0), torch.tensor(lens)).to(DEV) if by else \
        torch.zeros(T, dtype=torch.long, device=DEV)
    put = lambda x: torch.zeros((G, x.shape[1]), dtype=torch.float64,  # noqa: E731
                                device=DEV).index_put_((sg,), x, accumulate=True)
    counts, P, n = put(hot), put(p), put(m.double()[:, None])
    n1, S, N = n.clamp(min=1), int((n > 0).sum()), int(m.sum())
    f = counts / (k * n1)
    bal, zl = float(E * (f * P / n1).sum() / S), float(lse.square().sum() / N)
    held = torch.gather(p, 1, ids)
    # p = exp(z - max) / sum: differences of at most 20 rounded twice, E sums, a few 2^-24 more
    tol = (40 + 8 + np.log2(E) + 4) * 2.0 ** -24
    half = torch.finfo(dtype).eps / 2
    for norm in (True, False):
        prm = R.router_params(E, k, norm_topk=norm, balance_coef=cb, z_coef=cz, scope=scope)
        o = R.rft_router_fwd(tok, z, prm)
        st = R.stats_to_dict(o.stats, R.rft_router_stats)
        assert torch.equal(o.expert_ids, torch.where(m[:, None], ids, torch.full_like(ids, -1)).int())
        assert torch.equal(o.counts.double(), counts)
        assert (st["n_valid"], st["n_groups"], st["max_count"]) == (N, S, int(counts.max()))
        share = held.sum(1, keepdim=True).clamp(min=1e-300) if norm else torch.ones_like(held[:, :1])
        gates = held / share
        assert bool(((o.gates - gates).abs() <= 2 * tol * gates + 1e-37).all())
        assert bool(((o.lse - lse).abs() <= 2 * tol + 2.0 ** -23 * lse.abs()).all())
        for name, x in (("balance_loss", bal), ("z_loss", zl), ("loss", cb * bal + cz * zl)):
            assert abs(st[name] - x) <= 8 * tol * abs(x), name
        d = R.rft_router_bwd(tok, z, prm, o, d_gates=dg).double()
        own = dg.double()
        if norm:
            own = (own - (own * gates).sum(1, keepdim=True)) / share
        dp = (cb / S * E * f / n1)[sg] + torch.zeros_like(p).scatter_(1, ids, own * m[:, None])
        dz = p * (dp - (p * dp).sum(1, keepdim=True) + 2 * cz / N * lse[:, None])
        # what the subtractions cancel: the scale of a rounding of the gradient
        scale = p * (dp.abs() + (p * dp.abs()).sum(1, keepdim=True) + 2 * cz / N * lse[:, None].abs())
        if norm:
            scale += p * hot * ((dg.double() * gates).abs().sum(1, keepdim=True) / share)
        lim = 8 * tol * (1 + E ** 0.5 / 8) * scale + half * dz.abs() + 1e-37
        assert bool(((d - dz).abs() <= lim).all())

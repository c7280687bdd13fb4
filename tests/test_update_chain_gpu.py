"""A training step of a small policy with a mixture-of-experts layer, as a program runs it:
router forward, the experts' mixture, the policy head's fused step (d_hidden, d_weight),
the router's backward from the gates' gradients, the global norm over every gradient, the
orthogonalised update of the router's and the experts' matrices and AdamW on the head;
against the same step in float64 on the host."""
import numpy as np
import pytest
import torch

import paper_2505_17826_amd as R
from tests.gpu_cases import requires_gpu
from tests.test_ortho_gpu import LIMIT, polynomial

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")


def test_training_step():
    n_seq, pad, d, E, k, V = 8, 12, 64, 6, 2, 300
    T = n_seq * pad
    g = torch.Generator().manual_seed(0)
    rn = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    lens = torch.randint(1, pad + 1, (n_seq,), generator=g)
    lens[3] = 0
    mask = (torch.arange(pad)[None] < lens[:, None]).to(torch.uint8).view(-1)
    starts = (torch.arange(n_seq + 1) * pad).to(torch.int32)
    ids = torch.randint(0, V, (T,), generator=g).to(torch.int32)
    x, wr, we = rn(T, d), rn(E, d) / 8, rn(E, d, d) / 8
    head = 2 * rn(V, d) / 8
    old, ref = -5 + 0.1 * rn(T), -5 + 0.1 * rn(T)
    adv = rn(n_seq)
    cb, cz, lr, mu, max_norm = 0.1, 0.01, 0.02, 0.9, 0.05
    ppo = R.ppo_params(0.2, 0.2, 0.001, 0)

    # ---- the library's calls
    D = {q: v.to(DEV) for q, v in dict(x=x, wr=wr.clone(), we=we.clone(), head=head.clone(), old=old,
                                       ref=ref, adv=adv).items()}
    tok = R.Tokens(starts.to(DEV), mask.to(DEV), ids.to(DEV))
    prm = R.router_params(E, k, balance_coef=cb, z_coef=cz, scope=R.RFT_BALANCE_ROLLOUT)
    logits = D["x"] @ D["wr"].t()
    fwd = R.rft_router_fwd(tok, logits, prm)
    sel = fwd.expert_ids.clamp(min=0).long()
    y = torch.einsum("td,eod->teo", D["x"], D["we"])  # every expert, for the test's sake
    ys = torch.gather(y, 1, sel[:, :, None].expand(T, k, d))
    h = (fwd.gates[:, :, None] * ys).sum(1)
    logp, ent, lse, grad, dh, dhead, stats = R.rft_ppo_clip_step(tok, h, D["head"], D["old"],
                                                                 D["ref"], D["adv"], ppo)
    d_gates = (dh[:, None] * ys).sum(2)
    dl = R.rft_router_bwd(tok, logits, prm, fwd, d_gates=d_gates.contiguous())
    gr = dl.t() @ D["x"]
    hot = torch.zeros((T, E), device=DEV).scatter_(1, sel, fwd.gates)
    ge = torch.einsum("te,to,td->eod", hot, dh, D["x"])
    bufs = [torch.zeros_like(D["wr"]), torch.zeros_like(D["we"])]
    m, v = torch.zeros_like(D["head"]), torch.zeros_like(D["head"])
    every = R.Params([(None, t.contiguous(), None, None) for t in (gr, ge, dhead)])
    clip = R.rft_grad_norm(every, max_norm)
    mp = R.muon_params(lr, mu, True, 0.1, 1.0)
    R.rft_muon_step(D["wr"], gr.contiguous(), bufs[0], mp, clip=clip)
    R.rft_muon_step(D["we"], ge.contiguous(), bufs[1], mp, clip=clip)
    R.rft_adamw_step(R.Params([(D["head"], dhead, m, v)]), R.adamw_params(lr, step=1), clip=clip)
    torch.cuda.synchronize()

    # ---- the same in float64
    xd, wrd, wed = x.double(), wr.double().requires_grad_(), we.double().requires_grad_()
    z = xd @ wrd.t()
    p = torch.softmax(z, 1)
    on = mask.bool()
    sd = torch.argsort(z.detach(), dim=1, descending=True, stable=True)[:, :k]
    assert torch.equal(sd[on], sel.cpu()[on]) and bool((fwd.expert_ids.cpu()[~on] == -1).all())
    gates = torch.gather(p, 1, sd)
    gates = gates / gates.sum(1, keepdim=True) * on[:, None]
    yd = torch.einsum("td,eod->teo", xd, wed)
    hd = (gates[:, :, None] * torch.gather(yd, 1, sd[:, :, None].expand(T, k, d))).sum(1)
    # the surrogate and its KL term as the header states them
    eps, beta = float(np.float32(0.2)), float(np.float32(0.001))
    hh, wh = hd.detach().requires_grad_(), head.double().requires_grad_()
    lp = torch.log_softmax(hh @ wh.t(), 1).gather(1, ids.long()[:, None])[:, 0]
    A = adv.double().repeat_interleave(pad)
    rho = torch.exp(lp - old.double())
    pg = torch.maximum(-A * rho, -A * rho.clamp(1 - eps, 1 + eps))
    dk = ref.double() - lp
    per = pg + beta * (torch.expm1(dk) - dk)
    n = on.view(n_seq, pad).sum(1).clamp(min=1).repeat_interleave(pad)
    loss = (per * on / n).sum() / int((lens > 0).sum())
    loss.backward()
    dhd, dWd = hh.grad, wh.grad
    assert abs(R.stats_to_dict(stats)["loss"] - float(loss.detach())) <= 1e-5 * abs(float(loss.detach())) + 1e-8
    # balance and z-loss of each rollout
    hotd = torch.zeros((T, E), dtype=torch.float64).scatter_(1, sd, 1.0) * on[:, None]
    nn = on.view(n_seq, pad).sum(1).double()
    f = hotd.view(n_seq, pad, E).sum(1) / (k * nn.clamp(min=1)[:, None])
    P = (p * on[:, None]).view(n_seq, pad, E).sum(1) / nn.clamp(min=1)[:, None]
    bal = E * (f * P).sum() / int((nn > 0).sum())
    zl = ((torch.logsumexp(z, 1) ** 2) * on).sum() / int(on.sum())
    (cb * bal + cz * zl + (hd * dhd).sum()).backward()
    st = R.stats_to_dict(fwd.stats, R.rft_router_stats)
    assert abs(st["loss"] - float((cb * bal + cz * zl).detach())) <= 1e-5 * st["loss"]
    rel = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())  # noqa: E731
    assert rel(gr, wrd.grad) <= 1e-4 and rel(ge, wed.grad) <= 1e-4 and rel(dhead, dWd) <= 1e-4
    norm = torch.sqrt(wrd.grad.norm() ** 2 + wed.grad.norm() ** 2 + dWd.norm() ** 2)
    s = min(1.0, max_norm / float(norm))
    assert abs(float(clip.norm) - float(norm)) <= 1e-4 * float(norm)
    assert abs(float(clip.scale) - s) <= 1e-4 * s
    lim = LIMIT[R.RFT_PRODUCTS_THREE] + 141 * 1e-4  # the gradients' own error, amplified
    for got, w, gd in ((D["wr"], wr, wrd.grad), (D["we"], we, wed.grad)):
        u = s * (1 - mu) * (1 + mu) * gd
        step = lr * polynomial(u)
        want = w.double() * (1 - lr * 0.1) - step
        assert float((got.double().cpu() - want).norm()) <= lim * float(step.norm()) + 1e-6 * float(w.norm())
    # AdamW's first step is the sign of the gradient where that is not near eps
    gd = s * dWd
    want = head.double() * (1 - lr * 0.01) - lr * gd / (gd.abs() + 1e-8)
    sure = gd.abs() > 1e-3 * float(gd.abs().max())
    assert float((D["head"].double().cpu() - want)[sure].abs().max()) <= 1e-4 * lr + 1e-6

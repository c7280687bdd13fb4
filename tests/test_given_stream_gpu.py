"""Calls on a given stream allocate from that stream's memory (a block freed on the caller's
stream may still be in use by work pending there), and give the same results as the
caller's own stream."""
import pytest
import torch

import paper_2505_17826_amd as R
from tests.gpu_cases import requires_gpu

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")


def stream_of(t):
    """The stream whose memory holds t."""
    at = t.data_ptr()
    return next(s["stream"] for s in torch.cuda.memory_snapshot()
                if s["address"] <= at < s["address"] + s["total_size"])


def test_router_and_updates():
    T, E, k = 4096, 64, 4
    g = torch.Generator(DEV).manual_seed(3)
    z = torch.randn((T, E), generator=g, device=DEV)
    x = torch.randn((300, 700), generator=g, device=DEV)
    tok = R.Tokens(torch.tensor([0, 1000, T], dtype=torch.int32, device=DEV),
                   torch.ones(T, dtype=torch.uint8, device=DEV))
    prm = R.router_params(E, k, balance_coef=0.1, z_coef=0.1)
    ps = R.Params([(None, x, None, None)])

    def every(stream):
        o = R.rft_router_fwd(tok, z, prm, stream=stream)
        d = R.rft_router_bwd(tok, z, prm, o, stream=stream)
        clip = R.rft_grad_norm(ps, 1.0, stream=stream)
        q = R.rft_orthogonalize(x, R.muon_params(), stream=stream)
        w = x.clone()
        torch.cuda.synchronize()
        R.rft_muon_step(w, x, None, R.muon_params(), clip=clip, stream=stream)
        torch.cuda.synchronize()
        return [*R._arrays(o), d, clip.buf, q], w

    want, w0 = every(None)
    # blocks of every size that a call needs, freed on the caller's stream
    del want[:]
    side = torch.cuda.Stream()
    got, w1 = every(side)
    assert all(stream_of(t) == side.cuda_stream for t in got)
    want, _ = every(None)
    assert all(stream_of(t) == 0 for t in want)
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(w0, w1)


def test_the_policy_step():
    T, d, V = 64, 32, 200
    g = torch.Generator(DEV).manual_seed(4)
    h, w = (torch.randn(s, generator=g, device=DEV) / 6 for s in ((T, d), (V, d)))
    ids = torch.randint(0, V, (T,), generator=g, device=DEV).to(torch.int32)
    old, ref = (-5 + 0.1 * torch.randn(T, generator=g, device=DEV) for _ in range(2))
    adv = torch.randn(4, generator=g, device=DEV)
    tok = R.Tokens((torch.arange(5, device=DEV) * 16).to(torch.int32),
                   torch.ones(T, dtype=torch.uint8, device=DEV), ids)
    want = R.rft_ppo_clip_step(tok, h, w, old, ref, adv, R.ppo_params())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = R.rft_ppo_clip_step(tok, h, w, old, ref, adv, R.ppo_params(), stream=side)
    torch.cuda.synchronize()
    assert all(stream_of(t) == side.cuda_stream for t in got)
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))

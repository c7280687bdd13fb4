"""What an entry point allocates or clears when it is given a stream: with that stream current
(no GPU needed: the library and torch's streams are stand-ins).  Memory of the caller's current
stream may still be in use by work pending there, and a fill there would not be ordered
with the call."""
import contextlib
import types

import pytest
import torch

import paper_2505_17826_amd as R


class Stream:
    cuda_stream = 7
    device = torch.device("cpu")  # of the arrays here


@pytest.fixture
def spy(monkeypatch):
    """Records the stream current at every allocation and call, and the arrays recorded."""
    log = types.SimpleNamespace(current=None, allocated=[], called=[], recorded=[])

    @contextlib.contextmanager
    def stream(s):
        before, log.current = log.current, s
        yield
        log.current = before

    for name in ("empty", "zeros", "empty_like", "empty_strided", "zeros_like"):
        def make(*a, _f=getattr(torch, name), **k):
            log.allocated.append(log.current)
            return _f(*a, **k)
        monkeypatch.setattr(torch, name, make)

    class Lib:
        def __getattr__(self, name):
            def call(*a):
                if "bytes" in name:
                    return 64
                log.called.append(a[-1])
                return R.RFT_OK
            return call

    monkeypatch.setattr(R, "lib", Lib)
    monkeypatch.setattr(R, "_need_gpu", lambda *ts: None)
    monkeypatch.setattr(R, "_call", lambda fn, dev, s, *a: fn(*a, s and s.cuda_stream))
    monkeypatch.setattr(R, "_used_on", lambda s, *ts: log.recorded.extend(
        (s, t) for t in ts if t is not None))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: log.current or "callers")
    return log


def calls():
    T, d, V, E = 6, 8, 16, 4
    tok = R.Tokens(torch.tensor([0, 2, T], dtype=torch.int32), torch.ones(T, dtype=torch.uint8),
                   torch.zeros(T, dtype=torch.int32))
    row, adv, group = torch.zeros(T), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    h, w, z = torch.zeros(T, d), torch.zeros(V, d), torch.zeros(T, V)
    ppo, rp = R.ppo_params(), R.router_params(E, 2, balance_coef=0.1)
    rz = torch.zeros(T, E)
    fwd = R.RouterOut(torch.zeros(T, 2, dtype=torch.int32), torch.zeros(T, 2), row, torch.zeros(
        1, E, dtype=torch.int32), torch.zeros(1, E), torch.zeros(6))
    p = R.Params([(w, w, w, w)])
    return {
        "rft_group_advantages": lambda s: R.rft_group_advantages(adv, 2, stream=s),
        "rft_group_advantages_positional": lambda s: R.rft_group_advantages(adv, 2, 1e-6, None, s),
        "rft_group_advantages_ids": lambda s: R.rft_group_advantages_ids(
            adv, group, 1, stream=s),
        "rft_token_logprobs": lambda s: R.rft_token_logprobs(tok, h, w, stream=s),
        "rft_token_logprobs_from_logits": lambda s: R.rft_token_logprobs_from_logits(tok, z, stream=s),
        "rft_ppo_clip_loss_fwd": lambda s: R.rft_ppo_clip_loss_fwd(tok, V, row, row, row, adv, ppo, stream=s),
        "rft_ppo_clip_loss_bwd": lambda s: R.rft_ppo_clip_loss_bwd(tok, h, w, row, row, stream=s),
        "rft_ppo_clip_loss_bwd_logits": lambda s: R.rft_ppo_clip_loss_bwd_logits(tok, z, row, row, stream=s),
        "rft_ppo_clip_fused_logits": lambda s: R.rft_ppo_clip_fused_logits(
            tok, z, row, row, adv, ppo, stream=s),
        "rft_ppo_clip_step": lambda s: R.rft_ppo_clip_step(tok, h, w, row, row, adv, ppo, stream=s),
        "rft_sft_loss_fwd": lambda s: R.rft_sft_loss_fwd(tok, V, row, stream=s),
        "rft_dpo_loss_fwd": lambda s: R.rft_dpo_loss_fwd(tok, V, row, row, stream=s),
        "rft_router_fwd": lambda s: R.rft_router_fwd(tok, rz, rp, stream=s),
        "rft_router_fwd_alone": lambda s: R.rft_router_fwd(tok, rz, rp, want_loss=False, stream=s),
        "rft_router_bwd": lambda s: R.rft_router_bwd(tok, rz, rp, fwd, stream=s),
        "rft_grad_norm": lambda s: R.rft_grad_norm(p, stream=s),
        "rft_orthogonalize": lambda s: R.rft_orthogonalize(w, R.muon_params(), stream=s),
        "rft_muon_step": lambda s: R.rft_muon_step(w, w, None, R.muon_params(), stream=s),
    }


def prepared(spy, name):
    f = calls()[name]
    for log in (spy.allocated, spy.called, spy.recorded):
        log.clear()
    return f


def names():
    import re
    return re.findall(r'"(rft_\w+)": lambda', open(__file__).read())


@pytest.mark.parametrize("name", names())
def test_allocations_are_the_streams(spy, name):
    f, side = prepared(spy, name), Stream()
    out = f(side)
    assert spy.allocated and all(s is side for s in spy.allocated)
    assert len(spy.called) == 1 and getattr(spy.called[0], "value", spy.called[0]) == 7
    # every result is known to be read on the caller's stream
    for t in R._arrays(out):
        assert any(s == "callers" and x is t for s, x in spy.recorded)
    assert spy.current is None


@pytest.mark.parametrize("name", names())
def test_without_a_stream_nothing_changes(spy, name):
    if "positional" in name:
        return
    f = prepared(spy, name)
    spy.current = Stream()  # the caller's current one
    f(None)
    assert spy.allocated and all(s is spy.current for s in spy.allocated)
    assert not [s for s, _ in spy.recorded if s is not None]


def test_a_stream_of_another_device_is_refused(spy):
    side, x = Stream(), torch.zeros(2, device="meta")
    with pytest.raises(RuntimeError, match="meta"):
        R.rft_group_advantages(x, 2, stream=side)
    with pytest.raises(RuntimeError, match="meta"):
        R.rft_group_advantages(torch.zeros(2), 2, out=x, stream=side)
    assert not spy.called

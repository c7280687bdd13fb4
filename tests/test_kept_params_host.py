"""A kept Params follows its tensors (no GPU needed: the pointers that a call would get are
compared, nothing is launched): gradients that the backward pass made anew, storages that were
replaced."""
import pytest
import torch

import paper_2505_17826_amd as R


@pytest.fixture(autouse=True)
def host_tensors(monkeypatch):
    monkeypatch.setattr(R, "_need_gpu", lambda *ts: None)


@pytest.fixture
def passed(monkeypatch):
    """What each call passed to the library: the entries of the list."""
    seen = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: 64

    def call(fn, dev, stream, params, n, *a):
        seen.append([(p.weight, p.grad, p.m, p.v, p.master, p.n) for p in params[:n]])

    monkeypatch.setattr(R, "lib", Lib)
    monkeypatch.setattr(R, "_call", call)
    return seen


def entry(*ts):
    return tuple(None if t is None else t.data_ptr() for t in ts) + (ts[1].numel(),)


def backward(w):
    w.grad = None
    (w * torch.arange(w.numel(), dtype=w.dtype)).sum().backward()


def test_gradients_made_anew(passed):
    w = torch.ones(5000, requires_grad=True)
    w2, g2, m, v, m2, v2 = (torch.zeros(5000) for _ in range(6))
    backward(w)
    ps = R.Params([(w, w.grad, m, v), (w2, g2, m2, v2)])
    for i in range(3):
        R.rft_grad_norm(ps, 1.0)
        R.rft_adamw_step(ps, R.adamw_params(1e-3))
        want = [entry(w, w.grad, m, v, None), entry(w2, g2, m2, v2, None)]
        assert passed[-2:] == [want, want]
        old = w.grad  # held, so that its memory is not given out again
        backward(w)
        assert w.grad.data_ptr() != old.data_ptr()
    w.grad = None
    with pytest.raises(RuntimeError, match="tensor 0"):
        R.rft_adamw_step(ps, R.adamw_params(1e-3))
    w.grad = torch.zeros(5000)
    ps.now()
    w.data, w.grad = torch.zeros(10), torch.zeros(10)
    with pytest.raises(TypeError, match="tensor 0"):  # not the size of m and v
        ps.now()


def test_storages_replaced(passed):
    w, g, m, v = (torch.zeros(4000) for _ in range(4))
    ps = R.Params([(w.to(torch.bfloat16), g, m, v, w)])
    low = ps.tensors[0][0]
    for t in (low, g, m, v, w):
        t.data = torch.ones_like(t)
        R.rft_adamw_step(ps, R.adamw_params(1e-3))
        assert passed[-1] == [entry(low, g, m, v, w)]
    g.data = torch.ones(4000, dtype=torch.float64)
    with pytest.raises(TypeError):
        R.rft_adamw_step(ps, R.adamw_params(1e-3))

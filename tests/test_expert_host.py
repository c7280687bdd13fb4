"""The entry points of the experts on the host (no GPU needed): every bad argument gives its
status code before anything is enqueued, pointers are never read; what a given stream allocates;
and the float64 model that the GPU tests compare with, against differences."""
import ctypes

import pytest
import torch

import paper_2505_17826_amd as R
from tests import linear_model as M
from tests.test_given_stream_host import Stream, spy  # noqa: F401

FAKE = ctypes.c_void_p(0x1000)
BIG = 1 << 40


def _order(T=8, k=2, E=4, off=0x1000, slots=0x1000, places=0x1000):
    return R.rft_expert_order(T, k, E, off, slots, places)


def test_order_refusals():
    L = R.lib()
    calls = {
        "sort": lambda o, **a: L.rft_expert_sort(a.get("ids", FAKE), o, a.get("ws", FAKE),
                                                 a.get("nb", BIG), None),
        "gather": lambda o, **a: L.rft_expert_gather(o, a.get("x", FAKE), a.get("dt", 0), a.get("d", 8),
                                                     None, a.get("out", FAKE), None),
        "combine": lambda o, **a: L.rft_expert_combine(o, a.get("x", FAKE), a.get("dt", 0),
                                                       a.get("d", 8), None, None, a.get("out", FAKE), None),
        "bwd": lambda o, **a: L.rft_expert_combine_bwd(o, a.get("x", FAKE), a.get("rows", FAKE),
                                                       a.get("dt", 0), a.get("d", 8), None,
                                                       a.get("out", FAKE), a.get("dg", FAKE), None)}
    for name, f in calls.items():
        by = lambda *a, **kw: f(ctypes.byref(_order(*a, **kw)))  # noqa: E731
        assert f(None) == R.RFT_E_NULL, name
        for T, k, E in ((-1, 2, 4), (8, 0, 4), (8, 17, 4), (8, 2, 0), (8, 2, 1025), (1 << 30, 2, 4),
                        (1 << 62, 16, 4)):
            assert by(T, k, E) == R.RFT_E_SHAPE, (name, T, k, E)
        if name != "sort":
            o = ctypes.byref(_order())
            assert f(o, dt=2) == R.RFT_E_DTYPE
            assert f(o, d=0) == R.RFT_E_SHAPE and f(o, d=(1 << 24) + 1) == R.RFT_E_SHAPE
            assert f(o, x=None) == R.RFT_E_NULL
            assert by(places=None) == R.RFT_E_NULL
            assert f(ctypes.byref(_order(T=0, places=None)), x=None, out=None) == R.RFT_OK
    o = ctypes.byref(_order())
    assert calls["sort"](o, ids=None) == R.RFT_E_NULL
    for one in ("off", "slots", "places"):
        assert calls["sort"](ctypes.byref(_order(**{one: None}))) == R.RFT_E_NULL
    big = ctypes.byref(_order(T=100000))
    assert calls["sort"](big, ws=None) == R.RFT_E_WORKSPACE
    assert calls["sort"](big, nb=16) == R.RFT_E_WORKSPACE
    assert calls["gather"](o, out=None) == R.RFT_E_NULL and calls["combine"](o, out=None) == R.RFT_E_NULL
    assert calls["bwd"](o, rows=None) == R.RFT_E_NULL
    assert calls["bwd"](o, rows=None, out=None, dg=None) == R.RFT_OK
    assert L.rft_expert_sort_workspace_bytes(8, 2, 4) == 0
    assert L.rft_expert_sort_workspace_bytes(1 << 20, 8, 128) > 0
    assert L.rft_expert_sort_workspace_bytes(-1, 2, 4) == 0


def _groups(rows=16, E=2, off=0x1000, src=None, div=1, n=0):
    return R.rft_groups(rows, E, off, src, div, n)


def _fwd(g=None, x=FAKE, w=FAKE, dt=R.RFT_BF16, k=64, n=32, bias=None, act=0, res=None, y=FAKE, z=None,
         ws=FAKE, nb=BIG):
    g = _groups() if g is None else g
    return R.lib().rft_linear(ctypes.byref(g) if g else None, x, w, dt, k, n, bias, act, res, y, z, ws,
                              nb, None)


def _bwd(g=None, dy=FAKE, z=FAKE, x=FAKE, w=FAKE, dt=R.RFT_BF16, k=64, n=32, act=0, dx=FAKE, dw=FAKE,
         dwt=R.RFT_F32, db=FAKE, acc=0, ws=FAKE, nb=BIG):
    g = _groups() if g is None else g
    return R.lib().rft_linear_bwd(ctypes.byref(g) if g else None, dy, z, x, w, dt, k, n, act, dx, dw, dwt,
                                  db, acc, ws, nb, None)


def test_linear_refusals():
    for f in (_fwd, _bwd):
        assert f(g=False) == R.RFT_E_NULL
        assert f(g=_groups(off=None)) == R.RFT_E_NULL
        for kw in (dict(rows=-1), dict(rows=1 << 31), dict(E=0), dict(E=1025), dict(src=0x1000, div=0),
                   dict(src=0x1000, n=-1), dict(src=0x1000, n=1 << 31)):
            assert f(g=_groups(**kw)) == R.RFT_E_SHAPE, kw
        assert f(dt=2) == R.RFT_E_DTYPE
        assert f(act=4) == R.RFT_E_PARAM and f(act=-1) == R.RFT_E_PARAM
        for kw in (dict(k=0), dict(n=0), dict(k=-8), dict(k=(1 << 21) + 8), dict(n=(1 << 21) + 8),
                   dict(k=60), dict(n=36), dict(n=24, act=R.RFT_ACT_SWIGLU), dict(k=1 << 20, n=1 << 12),
                   dict(dt=R.RFT_F32, n=33, act=R.RFT_ACT_SWIGLU)):
            assert f(**kw) == R.RFT_E_SHAPE, kw
        assert f(g=_groups(src=0x1000, n=1 << 25)) == R.RFT_E_SHAPE  # source_rows k
        assert f(g=_groups(rows=(1 << 31) - 1), n=1 << 14) == R.RFT_E_SHAPE
        for one in ("x", "w"):
            assert f(**{one: None}) == R.RFT_E_NULL
            assert f(**{one: ctypes.c_void_p(0x1008)}) == R.RFT_E_SHAPE
    assert _fwd(y=None) == R.RFT_E_NULL
    for one in ("bias", "res", "y", "z"):
        assert _fwd(**{one: ctypes.c_void_p(0x1008)}) == R.RFT_E_SHAPE
    assert _fwd(g=_groups(rows=0), x=None, w=None, y=None) == R.RFT_OK
    for one in ("dy", "z", "dx", "dw"):
        assert _bwd(act=1, **{one: ctypes.c_void_p(0x1008)}) == R.RFT_E_SHAPE
    assert _bwd(dy=None) == R.RFT_E_NULL and _bwd(z=None, act=1) == R.RFT_E_NULL
    assert _bwd(dwt=3) == R.RFT_E_DTYPE and _bwd(dt=R.RFT_F32, dwt=R.RFT_BF16) == R.RFT_E_DTYPE
    assert _bwd(dwt=R.RFT_BF16, acc=1) == R.RFT_E_PARAM
    assert _bwd(act=1, ws=None) == R.RFT_E_WORKSPACE and _bwd(act=1, nb=64) == R.RFT_E_WORKSPACE
    assert _bwd(act=1, ws=ctypes.c_void_p(0x1008)) == R.RFT_E_WORKSPACE
    assert _bwd(dx=None, dw=None, db=None) == R.RFT_OK


def test_linear_workspaces():
    L = R.lib()
    size = lambda g, act=0, k=64, n=32, dt=R.RFT_BF16: L.rft_linear_bwd_workspace_bytes(  # noqa: E731
        ctypes.byref(g), dt, k, n, act)
    assert size(_groups(rows=4096), act=1) >= 4096 * 32 * 2  # dz
    assert size(_groups(rows=-1)) == 0 and size(_groups(), k=60) == 0
    assert L.rft_linear_workspace_bytes(None, R.RFT_BF16, 64, 32, 0) == 0


def _cpu_calls():
    ids = torch.zeros(6, 2, dtype=torch.int32)
    o = R.ExpertOrder(torch.zeros(5, dtype=torch.int32), torch.zeros(12, dtype=torch.int32), ids)
    x, rows, w = torch.zeros(6, 8), torch.zeros(12, 8), torch.zeros(4, 16, 8)
    dy = torch.zeros(12, 16)
    return {
        "sort": lambda s: R.rft_expert_sort(ids, 4, stream=s),
        "gather": lambda s: R.rft_expert_gather(o, x, stream=s),
        "combine": lambda s: R.rft_expert_combine(o, rows, stream=s),
        "combine_bwd": lambda s: R.rft_expert_combine_bwd(o, x, rows, stream=s),
        "linear": lambda s: R.rft_linear(x, w, groups=o.groups(gather=True), want_z=True, stream=s),
        "linear_bwd": lambda s: R.rft_linear_bwd(dy, x, w, groups=o.groups(gather=True),
                                                 want_db=True, stream=s)}


@pytest.mark.parametrize("name", list(_cpu_calls()))
def test_given_stream(spy, name):  # noqa: F811
    f, side = _cpu_calls()[name], Stream()
    for log in (spy.allocated, spy.called, spy.recorded):
        log.clear()
    out = f(side)
    assert spy.allocated and all(s is side for s in spy.allocated)
    assert spy.called == [7]
    for t in R._arrays(out):
        assert any(s == "callers" and x is t for s, x in spy.recorded)
    for log in (spy.allocated, spy.called, spy.recorded):
        log.clear()
    f(None)
    assert spy.allocated and all(s is None for s in spy.allocated)
    assert not [s for s, _ in spy.recorded if s is not None]


def test_binding_refusals(spy):  # noqa: F811
    i32 = dict(dtype=torch.int32)
    ids, x, rows, w = torch.zeros(6, 2, **i32), torch.zeros(6, 8), torch.zeros(12, 8), torch.zeros(4, 16, 8)
    o = R.ExpertOrder(torch.zeros(5, **i32), torch.zeros(12, **i32), ids)
    bad = [lambda: R.rft_expert_sort(ids.long(), 4), lambda: R.rft_expert_sort(ids[0], 4),
           lambda: R.rft_expert_sort(ids.t(), 4), lambda: R.rft_expert_sort(ids, 5, out=o),
           lambda: R.rft_expert_gather(o, rows), lambda: R.rft_expert_gather(o, x, out=rows.bfloat16()),
           lambda: R.rft_expert_gather(o, x, gates=torch.zeros(6, 3)),
           lambda: R.rft_expert_gather(o, x.half()), lambda: R.rft_expert_combine(o, x),
           lambda: R.rft_expert_combine(o, rows, residual=rows),
           lambda: R.rft_expert_combine(o, rows, gates=torch.zeros(6, 2).double()),
           lambda: R.rft_expert_combine_bwd(o, x, x),
           lambda: R.rft_linear(x, w.bfloat16(), groups=o.groups()),
           lambda: R.rft_linear(rows, w, groups=R.Groups(torch.zeros(4, **i32))),
           lambda: R.rft_linear(rows, w[0].t(), groups=None), lambda: R.rft_linear(x[:, ::2], w[0]),
           lambda: R.rft_linear(rows, w, groups=o.groups(), bias=torch.zeros(16)),
           lambda: R.rft_linear(rows, w, groups=o.groups(), residual=torch.zeros(12, 8)),
           lambda: R.rft_linear_bwd(torch.zeros(12, 8), rows, w, groups=o.groups()),
           lambda: R.rft_linear_bwd(torch.zeros(12, 16), rows, w, groups=o.groups(), accumulate=True),
           lambda: R.rft_linear_bwd(torch.zeros(12, 16), rows, w, groups=o.groups(),
                                    d_weight=w, dw_dtype=torch.bfloat16)]
    for i, f in enumerate(bad):
        with pytest.raises(TypeError):
            f()
            raise AssertionError(i)


def test_cpu_tensors_are_refused():
    x = torch.zeros(4, 8)
    with pytest.raises(RuntimeError):
        R.rft_linear(x, x)
    with pytest.raises(RuntimeError):
        R.rft_expert_sort(torch.zeros(4, 2, dtype=torch.int32), 4)


@pytest.mark.parametrize("act", M.ACTS)
def test_model_gradients_by_differences(act):
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, w, b, off = r(7, 5), r(3, 6, 5), r(3, 6), [0, 4, 4, 7]
    dy = r(7, 3 if act == "swiglu" else 6)
    _, z, _ = M.forward(x, w, b, act, None, off)
    dx, dw, db = M.backward(dy, z, x, w, act, off)[:3]
    h = 1e-5
    for t, grad in ((x, dx), (w, dw), (b, db)):
        for i in range(0, t.numel(), 3):
            old = float(t.view(-1)[i])
            v = []
            for s in (h, -h):
                t.view(-1)[i] = old + s
                v.append((M.forward(x, w, b, act, None, off)[0] * dy).sum())
            t.view(-1)[i] = old
            assert abs((v[0] - v[1]) / (2 * h) - grad.reshape(-1)[i]) < 1e-7

"""Refusals of the router and update entry points, on the host (no GPU needed): every bad
argument gives its status code before anything is enqueued; pointers are never read."""
import ctypes
import math

import pytest

import paper_2505_17826_amd as R

FAKE = ctypes.c_void_p(0x1000)


def _tok(T=8, n_seq=2, ss=0x1000, mask=0x1000):
    return R.rft_tokens(T, n_seq, ss, mask, None)


def _fwd(tok=None, logits=FAKE, dtype=R.RFT_F32, ld=64, p=None, ids=FAKE, gates=FAKE, lse=FAKE,
         counts=FAKE, dprob=FAKE, stats=FAKE, ws=FAKE, nb=1 << 30):
    tok = _tok() if tok is None else tok
    p = R.router_params(64, 4) if p is None else p
    return R.lib().rft_router_fwd(ctypes.byref(tok) if tok else None, logits, dtype, ld,
                                  ctypes.byref(p) if p else None, ids, gates, lse, counts, dprob,
                                  stats, ws, nb, None)


def _bwd(tok=None, logits=FAKE, dtype=R.RFT_F32, ld=64, p=None, ids=FAKE, lse=FAKE, dg=FAKE,
         dprob=FAKE, stats=FAKE, dl=ctypes.c_void_p(0x9000), ldd=64):
    tok = _tok() if tok is None else tok
    p = R.router_params(64, 4) if p is None else p
    return R.lib().rft_router_bwd(ctypes.byref(tok) if tok else None, logits, dtype, ld,
                                  ctypes.byref(p) if p else None, ids, lse, dg, dprob, stats, dl,
                                  ldd, None)


def test_router_refusals():
    for f in (_fwd, _bwd):
        assert f(tok=False) == R.RFT_E_NULL
        assert f(p=False) == R.RFT_E_NULL
        assert f(tok=_tok(T=-1)) == R.RFT_E_SHAPE
        assert f(tok=_tok(T=(1 << 30) + 1)) == R.RFT_E_SHAPE
        assert f(tok=_tok(n_seq=0)) == R.RFT_E_SHAPE
        assert f(tok=_tok(ss=None)) == R.RFT_E_NULL
        assert f(tok=_tok(mask=None)) == R.RFT_E_NULL
        assert f(logits=None) == R.RFT_E_NULL
        assert f(dtype=5) == R.RFT_E_DTYPE
        assert f(ld=63) == R.RFT_E_SHAPE
        for E, k in ((0, 1), (1025, 4), (64, 0), (64, 17), (8, 9), (-3, 1)):
            assert f(p=R.router_params(E, k), ld=2048) == R.RFT_E_SHAPE, (E, k)
        assert f(p=R.router_params(64, 4, scope=2)) == R.RFT_E_PARAM
        for c in (-1.0, math.inf, math.nan):
            assert f(p=R.router_params(64, 4, balance_coef=c)) == R.RFT_E_PARAM
            assert f(p=R.router_params(64, 4, z_coef=c)) == R.RFT_E_PARAM
        assert f(ids=None) == R.RFT_E_NULL
    assert _fwd(gates=None) == R.RFT_E_NULL
    for one in ("counts", "dprob", "stats"):
        assert _fwd(**{one: None}) == R.RFT_E_NULL
    assert _fwd(lse=None) == R.RFT_E_NULL
    assert _fwd(ws=None) == R.RFT_E_WORKSPACE and _fwd(nb=64) == R.RFT_E_WORKSPACE
    assert _fwd(ws=ctypes.c_void_p(0x1008)) == R.RFT_E_WORKSPACE
    huge = _tok(T=1 << 30, n_seq=1 << 30)
    assert _fwd(tok=huge, p=R.router_params(64, 4, scope=R.RFT_BALANCE_ROLLOUT)) == R.RFT_E_SHAPE
    for one in ("lse", "dprob", "stats", "dl"):
        assert _bwd(**{one: None}) == R.RFT_E_NULL
    assert _bwd(ldd=63) == R.RFT_E_SHAPE
    assert _bwd(ld=80, dl=FAKE, ldd=64) == R.RFT_E_SHAPE  # in place with another stride
    assert _bwd(tok=_tok(T=0, n_seq=0, mask=None), logits=None, ids=None, lse=None, dl=None) == R.RFT_OK


def test_router_workspace():
    L = R.lib()
    size = lambda T, n, **kw: L.rft_router_workspace_bytes(  # noqa: E731
        ctypes.byref(_tok(T, n)), ctypes.byref(R.router_params(128, 8, **kw)))
    assert 0 < size(1, 1) <= size(4096, 4) <= size(262144, 256)
    by = dict(scope=R.RFT_BALANCE_ROLLOUT)
    assert size(262144, 256, **by) > size(262144, 256)
    # rollouts of one row: a slot per wave and rollout, 8 bytes per expert
    assert size(1000, 1000, **by) >= 1000 * 128 * 8
    assert L.rft_router_workspace_bytes(None, ctypes.byref(R.router_params(8, 1))) == 0
    assert L.rft_router_workspace_bytes(ctypes.byref(_tok()), ctypes.byref(R.router_params(0, 1))) == 0


def _list(n=10, count=1, **null):
    a = (R.rft_param * count)()
    for i in range(count):
        d = dict(weight=0x1000, grad=0x2000, m=0x3000, v=0x4000, master=None)
        d.update(null)
        a[i] = R.rft_param(d["weight"], d["grad"], d["m"], d["v"], d["master"], n)
    return a


def test_update_refusals():
    L = R.lib()
    norm = lambda a, n, dt=R.RFT_F32, mx=1.0, clip=FAKE, ws=FAKE, nb=1 << 20: \
        L.rft_grad_norm(a, n, dt, mx, clip, ws, nb, None)  # noqa: E731
    assert norm(_list(), -1) == R.RFT_E_SHAPE
    assert norm(None, 1) == R.RFT_E_NULL
    assert norm(_list(n=-1), 1) == R.RFT_E_SHAPE
    assert norm(_list(n=1 << 41), 1) == R.RFT_E_SHAPE
    assert norm(_list(grad=None), 1) == R.RFT_E_NULL
    assert norm(_list(), 1, dt=7) == R.RFT_E_DTYPE
    for mx in (-1.0, math.inf, math.nan):
        assert norm(_list(), 1, mx=mx) == R.RFT_E_PARAM
    assert norm(_list(), 1, clip=None) == R.RFT_E_NULL
    assert norm(_list(n=1 << 20), 1, nb=8) == R.RFT_E_WORKSPACE
    assert norm(_list(), 1, ws=None) == R.RFT_E_WORKSPACE
    assert L.rft_grad_norm_workspace_bytes(_list(n=1 << 20, count=3), 3) == 3 * 32 * 8
    assert L.rft_grad_norm_workspace_bytes(_list(n=-2), 1) == 0
    assert L.rft_grad_norm_workspace_bytes(None, 2) == 0

    def step(a=None, n=1, w=R.RFT_F32, g=R.RFT_F32, **h):
        kw = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, step=1)
        kw.update(h)
        a = _list() if a is None else a
        return L.rft_adamw_step(a, n, w, g, ctypes.byref(R.adamw_params(**kw)), None, None)

    assert step(n=-1) == R.RFT_E_SHAPE
    for one in ("weight", "grad", "m", "v"):
        assert step(_list(**{one: None})) == R.RFT_E_NULL
    assert step(w=3) == R.RFT_E_DTYPE and step(g=3) == R.RFT_E_DTYPE
    for kw in (dict(lr=math.nan), dict(lr=math.inf), dict(weight_decay=math.inf), dict(beta1=1.0),
               dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=-1e-8),
               dict(eps=math.nan), dict(step=0)):
        assert step(**kw) == R.RFT_E_PARAM, kw
    assert step(_list(master=0x5000)) == R.RFT_E_PARAM  # a master of an fp32 weight
    assert L.rft_adamw_step(_list(), 1, 0, 0, None, None, None) == R.RFT_E_NULL
    assert step(_list(n=0)) == R.RFT_OK and step(n=0) == R.RFT_OK  # nothing to do, nothing enqueued


def test_binding_refuses_what_the_library_cannot_see():
    import torch
    t = torch.zeros(4)
    with pytest.raises(RuntimeError):
        R.Params([(t, t, t, t)])
    with pytest.raises(RuntimeError):
        R.rft_router_fwd(R.Tokens(torch.zeros(2, dtype=torch.int32), torch.ones(4, dtype=torch.uint8)),
                         torch.zeros(4, 8), R.router_params(8, 2))


def _mats(batch=1, rows=8, cols=16, rs=16, bs=128):
    return R.rft_matrices(batch, rows, cols, rs, bs)


def _ortho(m=None, g=FAKE, dt=R.RFT_F32, p=None, out=FAKE, odt=R.RFT_F32, ws=FAKE, nb=1 << 40):
    m = _mats() if m is None else m
    p = R.muon_params() if p is None else p
    return R.lib().rft_orthogonalize(ctypes.byref(m) if m else None, g, dt,
                                     ctypes.byref(p) if p else None, out, odt, ws, nb, None)


def _muon(m=None, g=FAKE, dt=R.RFT_F32, p=None, buf=FAKE, w=FAKE, wdt=R.RFT_F32, master=None,
          ws=FAKE, nb=1 << 40):
    m = _mats() if m is None else m
    p = R.muon_params() if p is None else p
    return R.lib().rft_muon_step(ctypes.byref(m) if m else None, g, dt, buf, w, wdt, master,
                                 ctypes.byref(p) if p else None, None, ws, nb, None)


def test_orthogonalize_refusals():
    for f in (_ortho, _muon):
        assert f(m=False) == R.RFT_E_NULL and f(p=False) == R.RFT_E_NULL
        assert f(g=None) == R.RFT_E_NULL
        for bad in (_mats(batch=-1), _mats(batch=65536), _mats(rows=0), _mats(cols=0),
                    _mats(rs=15), _mats(batch=2, bs=127), _mats(rows=16385, cols=16385, rs=16385),
                    _mats(rows=4, cols=(1 << 20) + 1, rs=1 << 21), _mats(rs=1 << 41)):
            assert f(m=bad) == R.RFT_E_SHAPE
        assert f(dt=2) == R.RFT_E_DTYPE
        for kw in (dict(steps=0), dict(steps=33), dict(eps=-1.0), dict(eps=math.nan),
                   dict(scale=math.inf), dict(coefs=(math.nan, 0, 0)), dict(products=2)):
            assert f(p=R.muon_params(**kw)) == R.RFT_E_PARAM, kw
        assert f(ws=None) == R.RFT_E_WORKSPACE and f(nb=4096) == R.RFT_E_WORKSPACE
        assert f(ws=ctypes.c_void_p(0x1004)) == R.RFT_E_WORKSPACE
        assert f(m=_mats(batch=0)) == R.RFT_OK  # nothing to do, nothing enqueued
    assert _ortho(out=None) == R.RFT_E_NULL and _ortho(odt=9) == R.RFT_E_DTYPE
    assert _ortho(dt=R.RFT_BF16) == R.RFT_E_PARAM  # in place with another type
    assert _muon(w=None) == R.RFT_E_NULL and _muon(wdt=9) == R.RFT_E_DTYPE
    assert _muon(master=FAKE) == R.RFT_E_PARAM  # a master of an fp32 weight
    for kw in (dict(lr=math.nan), dict(weight_decay=math.inf), dict(momentum=1.0),
               dict(momentum=-0.5), dict(momentum=math.nan)):
        assert _muon(p=R.muon_params(**kw)) == R.RFT_E_PARAM, kw


def test_orthogonalize_workspace():
    L = R.lib()
    size = lambda m, dt=R.RFT_F32, **kw: L.rft_orthogonalize_workspace_bytes(  # noqa: E731
        ctypes.byref(m), ctypes.byref(R.muon_params(**kw)), dt)
    one, three = size(_mats(), products=R.RFT_PRODUCTS_ONE), size(_mats(), products=R.RFT_PRODUCTS_THREE)
    # up to 128 rows only X is in memory, as hi + lo for either kind of products
    assert 0 < one <= three == size(_mats()) and size(_mats(), R.RFT_BF16) == one
    big = _mats(rows=300, cols=700, rs=700)
    assert size(big, products=R.RFT_PRODUCTS_ONE) < size(big, products=R.RFT_PRODUCTS_THREE) == size(big)
    assert size(big, R.RFT_BF16) == size(big, products=R.RFT_PRODUCTS_ONE)
    assert size(_mats(batch=4)) > 3 * three
    # the orientation does not matter
    assert size(_mats(rows=300, cols=700, rs=700)) == size(_mats(rows=700, cols=300, rs=300))
    assert size(_mats(rows=0)) == 0 and size(_mats(), 5) == 0 and size(_mats(), steps=0) == 0


def test_binding_refuses_other_layouts():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("device tensors")
    w = torch.zeros(8, 16, device="cuda")
    with pytest.raises(TypeError):
        R.rft_muon_step(w, torch.zeros(16, 8, device="cuda").t(), None, R.muon_params())
    with pytest.raises(TypeError):
        R.rft_muon_step(w, w.clone(), w.double(), R.muon_params())
    with pytest.raises(TypeError):
        R.rft_orthogonalize(w.t(), R.muon_params())


def test_new_kernels_have_no_spills(tmp_path):
    """Rows, accumulator tiles and lists held in vector registers stay there (scalar ones may
    be kept in lanes of vector registers)."""
    import os
    import shutil
    import subprocess
    from paper_2505_17826_amd import build_lib as B
    from tests.test_spills_host import _KERNEL
    hipcc = B.HIPCC if os.path.exists(B.HIPCC) else shutil.which("hipcc")
    if not hipcc:
        pytest.skip("hipcc not available")
    for src in ("k_router.hip", "k_adamw.hip", "k_ortho.hip"):
        out = tmp_path / (src + ".s")
        cmd = [hipcc, *[f for f in B.CFLAGS if f != "-fPIC"], *B.SOURCE_FLAGS.get(src, []),
               "--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o", str(out)]
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
        assert r.returncode == 0, r.stderr[-2000:]
        kernels = _KERNEL.findall(out.read_text())
        assert kernels and not [k for k in kernels if int(k[1]) or int(k[3])]

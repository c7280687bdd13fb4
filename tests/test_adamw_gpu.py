"""rft_grad_norm and rft_adamw_step against plain float64 arithmetic: types, masters,
unaligned and ragged tensors, lists longer than a launch holds, clipping, gradients that
are not finite, and what lies beside the tensors."""
import math

import numpy as np
import pytest
import torch

import paper_2505_17826_amd as R
from tests.gpu_cases import requires_gpu

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")
HYP = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=7)


def tensors(sizes, wdt, gdt, master, seed=0, offset=0):
    """Views of `sizes` elements into guarded buffers, `offset` elements from their start."""
    g = torch.Generator(DEV).manual_seed(seed)

    def one(n, dt, f):
        buf = torch.full((offset + n + 8,), 13.0, dtype=dt, device=DEV)
        buf[offset:offset + n] = f(torch.randn(n, generator=g, device=DEV)).to(dt)
        return buf, buf[offset:offset + n]

    out = []
    for n in sizes:
        w32 = 0.3 * torch.randn(n, generator=g, device=DEV)
        w = one(n, wdt, lambda x: w32)
        gr = one(n, gdt, lambda x: 0.01 * x)
        m = one(n, torch.float32, lambda x: 0.001 * x)
        v = one(n, torch.float32, lambda x: 1e-5 * x * x)
        ms = one(n, torch.float32, lambda x: w32) if master else (None, None)
        out.append((w, gr, m, v, ms))
    return out


def run(ts, max_norm=0.0, hyp=HYP, clip=True):
    ps = R.Params([tuple(x[1] for x in t) for t in ts])
    c = R.rft_grad_norm(ps, max_norm) if clip else None
    R.rft_adamw_step(ps, R.adamw_params(**hyp), clip=c)
    torch.cuda.synchronize()
    return c


def expect(before, scale, hyp):
    w, g, m, v, ms = [None if x is None else x.double() for x in before]
    b1, b2, lr, eps, wd = (hyp[q] for q in ("beta1", "beta2", "lr", "eps", "weight_decay"))
    g = g * scale
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    base = w if ms is None else ms
    return (base * (1 - lr * wd) - lr * (m / (1 - b1 ** hyp["step"])) /
            ((v / (1 - b2 ** hyp["step"])).sqrt() + eps), m, v)


@pytest.mark.parametrize("wdt,master", [(torch.float32, False), (torch.bfloat16, False),
                                        (torch.bfloat16, True)])
@pytest.mark.parametrize("gdt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1, 2, 4])
def test_step(wdt, master, gdt, offset):
    sizes = [1, 3, 4, 1000, 8192, 8193, 40001, 0]
    ts = tensors(sizes, wdt, gdt, master, seed=offset, offset=offset)
    before = [tuple(None if x[1] is None else x[1].clone() for x in t) for t in ts]
    total = math.sqrt(sum(float(b[1].double().square().sum()) for b in before))
    for max_norm in (0.0, total / 3, total * 2):
        for t, b in zip(ts, before):
            for x, y in zip(t, b):
                if y is not None:
                    x[1].copy_(y)
        c = run(ts, max_norm)
        # float32 of a float64 sum: one rounding each, the factor of one more division
        assert abs(float(c.norm) - total) <= 2.0 ** -23 * total and int(c.finite) == 1
        scale = min(1.0, float(np.float32(max_norm)) / total) if max_norm else 1.0
        assert abs(float(c.scale) - scale) <= 2.0 ** -23 * scale
        for t, b in zip(ts, before):
            w, m, v = expect(b, float(c.scale), HYP)
            # m, v: three roundings of terms no larger than the larger of their two summands
            # (scale g, the product, the sum; v one more), each 2^-24
            gm = b[1].double().abs() * scale
            assert bool(((t[2][1].double() - m).abs() <= 4 * 2.0 ** -24 * (b[2].double().abs() + gm)).all())
            assert bool(((t[3][1].double() - v).abs() <= 6 * 2.0 ** -24 * (b[3].double().abs() + gm * gm)).all())
            # w: its own roundings (two of |w|), and the step's, whose m carries an absolute
            # error as above and whose other factors carry 8 x 2^-24 relative
            base = (b[0] if b[4] is None else b[4]).double()
            hat = (v / (1 - 0.95 ** 7)).sqrt() + 1e-8
            lim = 2.0 ** -24 * (3 * base.abs() + 3e-3 / (1 - 0.9 ** 7) *
                                (12 * m.abs() + 4 * (b[2].double().abs() + gm)) / hat)
            got = t[0][1] if b[4] is None else t[4][1]
            extra = w.abs() * 2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0
            assert bool(((got.double() - w).abs() <= lim + extra).all())
            if master:
                assert torch.equal(t[0][1], t[4][1].to(wdt))
            for x in t:
                if x[0] is not None:  # nothing beside the tensor has changed
                    o = x[0].double()
                    assert bool((o[:offset] == 13).all()) and bool((o[offset + t[0][1].numel():] == 13).all())


def test_many_tensors_take_several_launches():
    sizes = [1 + 37 * i % 501 for i in range(101)]
    ts = tensors(sizes, torch.float32, torch.float32, False, seed=3)
    before = [tuple(None if x[1] is None else x[1].clone() for x in t) for t in ts]
    c = run(ts, 0.5)
    total = math.sqrt(sum(float(b[1].double().square().sum()) for b in before))
    assert abs(float(c.norm) - total) <= 2.0 ** -23 * total
    for t, b in zip(ts, before):
        w, m, v = expect(b, float(c.scale), HYP)
        assert float((t[0][1].double() - w).abs().max()) <= 1e-6
    assert R.rft_grad_norm(R.Params([]), 1.0).norm.item() == 0.0


def test_large_values_and_gradients_that_are_not_finite():
    for bad in (math.inf, -math.inf, math.nan):
        ts = tensors([1000, 70000], torch.bfloat16, torch.float32, True, seed=4)
        ts[1][1][1][69999] = bad
        before = [tuple(x[1].clone() for x in t) for t in ts]
        c = run(ts, 1.0)
        assert int(c.finite) == 0
        for t, b in zip(ts, before):
            for x, y in zip(t, b):
                assert torch.equal(x[1].view(torch.uint8), y.view(torch.uint8))
    ts = tensors([4096], torch.float32, torch.float32, False, seed=5)
    ts[0][1][1].fill_(1e30)  # squares past fp32
    c = run(ts, 1.0)
    assert int(c.finite) == 1 and abs(float(c.norm) / 64e30 - 1) <= 2.0 ** -22
    assert bool(torch.isfinite(ts[0][0][1]).all())
    ts[0][1][1].fill_(1e-30)  # squares below fp32
    c = R.rft_grad_norm(R.Params([tuple(x[1] for x in ts[0])]))
    assert abs(float(c.norm) / 64e-30 - 1) <= 2.0 ** -22


def test_norm_is_the_same_from_run_to_run_and_in_a_graph():
    ts = tensors([300001, 12345], torch.float32, torch.bfloat16, False, seed=6)
    ps = R.Params([tuple(x[1] for x in t) for t in ts])
    a, b = R.rft_grad_norm(ps, 0.1), R.rft_grad_norm(ps, 0.1)
    assert torch.equal(a.buf, b.buf)
    start = [t[0][1].clone() for t in ts]
    state = [[x[1].clone() for x in t[2:4]] for t in ts]

    def reset():
        for t, w, (m, v) in zip(ts, start, state):
            t[0][1].copy_(w), t[2][1].copy_(m), t[3][1].copy_(v)

    hyp = R.adamw_params(**HYP)
    for _ in range(3):
        R.rft_adamw_step(ps, hyp, clip=R.rft_grad_norm(ps, 0.1))
    want = [t[0][1].clone() for t in ts]
    reset()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c = R.rft_grad_norm(ps, 0.1)
        R.rft_adamw_step(ps, hyp, clip=c)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.buf, a.buf)
    for t, w in zip(ts, want):
        assert torch.equal(t[0][1], w)

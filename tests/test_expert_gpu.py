"""rft_expert_sort, rft_expert_gather, rft_expert_combine and rft_expert_combine_bwd against a
plain implementation: orders exactly, rows by the rounding of their types, over sizes around the
kernels' blocks, experts without slots, tokens without experts, repeated experts and odd rows."""
import math

import numpy as np
import pytest
import torch

import paper_2505_17826_amd as R
from tests.gpu_cases import requires_gpu

pytestmark = [pytest.mark.gpu, requires_gpu]
DEV = torch.device("cuda")
BF, F32 = torch.bfloat16, torch.float32


def reference(ids, E):
    flat = ids.reshape(-1)
    valid = (flat >= 0) & (flat < E)
    order = np.argsort(np.where(valid, flat, E), kind="stable")[:int(valid.sum())]
    slots = np.full(flat.size, -1)
    slots[:order.size] = order
    places = np.full(flat.size, -1)
    places[order] = np.arange(order.size)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[valid], minlength=E))])
    return offsets, slots, places.reshape(ids.shape)


def choose(T, E, k, seed, some=0.9, low=-2):
    r = np.random.default_rng(seed)
    ids = r.integers(0, E, size=(T, k))
    if E > 4:
        ids = np.where(r.random((T, k)) < 0.3, ids % 3, ids)  # an uneven load
    out = r.random((T, k)) >= some
    return np.where(out, r.choice([-1, low, E, E + 7, 2 ** 31 - 1, -2 ** 31], size=(T, k)), ids).astype(np.int32)


def sort(ids, E):
    o = R.rft_expert_sort(torch.from_numpy(ids).to(DEV), E)
    return o, [t.cpu().numpy() for t in (o.offsets, o.slots, o.places)]


# slots: none, one, around a wave, a block's 16 waves, the one-block limit, many blocks
@pytest.mark.parametrize("T,k", [(0, 2), (1, 1), (1, 8), (63, 1), (64, 1), (65, 1), (128, 8), (1023, 1),
                                 (1025, 3), (4096, 4), (4097, 4), (5000, 10), (40000, 8), (70001, 1)])
@pytest.mark.parametrize("E", (1, 2, 60, 128, 1000, 1024))
def test_sort(T, k, E):
    ids = choose(T, E, k, T + E)
    _, got = sort(ids, E)
    for a, b, name in zip(got, reference(ids, E), ("offsets", "slots", "places")):
        assert np.array_equal(a, b), name


def test_sort_extremes():
    for ids in (np.full((3000, 8), 5, np.int32), np.full((3000, 8), -1, np.int32),
                np.tile(np.arange(8, dtype=np.int32), (30000, 1))):
        _, got = sort(ids, 16)
        for a, b in zip(got, reference(ids, 16)):
            assert np.array_equal(a, b)


def make(T, E, k, d, dt, seed=0, some=0.9):
    ids = choose(T, E, k, seed, some)
    o, (offsets, slots, places) = sort(ids, E)
    g = torch.Generator().manual_seed(seed)
    n = T * k
    x, rows = torch.randn(T, d, generator=g).to(dt), torch.randn(n, d, generator=g).to(dt)
    gates = torch.rand(T, k, generator=g)
    return o, int(offsets[-1]), slots, places, x, rows, gates


ROWS = [(1, 4, 1, 8), (1, 16, 8, 1536), (5, 4, 2, 7), (33, 60, 4, 512), (200, 64, 8, 520), (130, 3, 16, 1),
        (64, 1, 1, 4104), (1000, 128, 3, 65)]


@pytest.mark.parametrize("dt", (BF, F32))
@pytest.mark.parametrize("gated", (False, True))
@pytest.mark.parametrize("T,E,k,d", ROWS)
def test_rows(T, E, k, d, dt, gated):
    o, n, slots, places, x, rows, gates = make(T, E, k, d, dt, seed=T + d)
    half = torch.finfo(dt).eps / 2
    G = gates.to(DEV) if gated else None
    one = gates if gated else torch.ones_like(gates)
    token = torch.from_numpy(slots[:n] // k)
    weight = one.reshape(-1)[torch.from_numpy(slots[:n])].double()[:, None]

    # gather: one product, one rounding (fp32: the same rounding; without gates a copy)
    buf = torch.full((T * k, d), 7.0, dtype=dt, device=DEV)
    got = R.rft_expert_gather(o, x.to(DEV), gates=G, out=buf).cpu().double()
    want = weight * x.double()[token]
    tol = (half + 2.0 ** -24) * want.abs() if gated else 0 * want
    assert ((got[:n] - want).abs() <= tol).all()
    assert (got[n:] == 7).all()

    # combine: k products and sums in fp32, one rounding; NaN rows of no token are not read
    rows[n:] = math.nan
    res = torch.randn(T, d, generator=torch.Generator().manual_seed(1)).to(dt)
    has = torch.from_numpy(places >= 0)[..., None]
    y = torch.where(has, rows.double()[torch.from_numpy(places).clamp(min=0)], torch.zeros(()).double())
    for residual in (None, res):
        got = R.rft_expert_combine(o, rows.to(DEV), gates=G,
                                   residual=None if residual is None else residual.to(DEV)).cpu().double()
        terms = one.double()[..., None] * y
        want, mag = terms.sum(1), terms.abs().sum(1)
        if residual is not None:
            want, mag = want + residual.double(), mag + residual.double().abs()
        tol = (k + 2) * 2.0 ** -24 * mag
        assert ((got - want).abs() <= tol + half * (want.abs() + tol)).all()

    # its backward
    do = torch.randn(T, d, generator=torch.Generator().manual_seed(2)).to(dt)
    buf = torch.full((T * k, d), 7.0, dtype=dt, device=DEV)
    dr, dg = R.rft_expert_combine_bwd(o, do.to(DEV), rows.to(DEV), gates=G, d_rows=buf)
    want = weight * do.double()[token]
    tol = (half + 2.0 ** -24) * want.abs() if gated else 0 * want
    assert ((dr.cpu().double()[:n] - want).abs() <= tol).all()
    assert (dr.cpu()[n:] == 7).all()
    want, mag = (do.double()[:, None] * y).sum(2), (do.double()[:, None] * y).abs().sum(2)
    assert ((dg.cpu().double() - want).abs() <= (d + 2) * 2.0 ** -24 * mag).all()
    assert (dg.cpu()[torch.from_numpy(places < 0)] == 0).all()

    # in place, and each alone
    R_ = rows.to(DEV).clone()
    dr2, dg2 = R.rft_expert_combine_bwd(o, do.to(DEV), R_, gates=G, d_rows=R_)
    assert torch.equal(dr2[:n], dr[:n]) and torch.equal(dg2, dg)
    only, none = R.rft_expert_combine_bwd(o, do.to(DEV), None, gates=G, want_d_gates=False)
    assert none is None and torch.equal(only[:n], dr[:n])
    none, only = R.rft_expert_combine_bwd(o, do.to(DEV), rows.to(DEV), gates=G, want_d_rows=False)
    assert none is None and torch.equal(only, dg)
    out = res.to(DEV).clone()
    a = R.rft_expert_combine(o, rows.to(DEV), gates=G, residual=res.to(DEV))
    assert torch.equal(a, R.rft_expert_combine(o, rows.to(DEV), gates=G, residual=out, out=out))


def test_values_of_slots_without_an_expert_do_not_count():
    """Gates of inf and NaN where there is no expert, NaN in rows of no slot."""
    o, n, slots, places, x, rows, gates = make(40, 8, 4, 24, F32, seed=3, some=0.5)
    gates[torch.from_numpy(places < 0)] = math.nan
    rows[n:] = math.inf
    out = R.rft_expert_combine(o, rows.to(DEV), gates=gates.to(DEV))
    assert torch.isfinite(out).all()
    none = torch.from_numpy((places < 0).all(1))
    assert (out.cpu()[none] == 0).all()


def test_an_order_of_other_sizes_stays_inside():
    """Places outside the rows are slots without an expert."""
    o, n, slots, places, x, rows, gates = make(20, 4, 2, 16, F32)
    o.places.fill_(40)
    o.places[3, 1] = -2 ** 31
    assert not R.rft_expert_combine(o, rows.to(DEV)).any()
    buf = torch.full((42 * 16,), 7.0, device=DEV)
    R.rft_expert_gather(o, x.to(DEV), out=buf[16:41 * 16].view(40, 16))
    assert (buf == 7).all()


def test_gradient_of_gather_by_differences():
    """fp32, linear in x: <c, gather(x + v) - gather(x)> = <combine(c), v>."""
    o, n, slots, places, x, rows, gates = make(50, 6, 3, 40, F32, seed=5)
    c = rows.to(DEV)
    c[n:] = 0
    v = torch.randn(50, 40, generator=torch.Generator().manual_seed(8))
    zero = lambda: torch.zeros(150, 40, device=DEV)  # noqa: E731
    for G in (None, gates.to(DEV)):
        a = R.rft_expert_gather(o, (x + v).to(DEV), gates=G, out=zero()).double()
        b = R.rft_expert_gather(o, x.to(DEV), gates=G, out=zero()).double()
        got = ((a - b) * c.double()).sum()
        want = (R.rft_expert_combine(o, c, gates=G).double() * v.to(DEV).double()).sum()
        # 6000 terms rounded by 2^-23 of their few units, random signs
        assert abs(float(got - want)) <= 6000 * 2.0 ** -22 * 4


def test_streams_and_graphs():
    T, E, k, d = 3000, 20, 8, 264  # past the one-block sort
    ids = torch.from_numpy(choose(T, E, k, 1)).to(DEV)
    x = torch.randn(T, d, device=DEV).to(BF)
    gates = torch.rand(T, k, device=DEV)

    def call(stream=None):
        o = R.rft_expert_sort(ids, E, stream=stream)
        rows = R.rft_expert_gather(o, x, stream=stream)
        out = R.rft_expert_combine(o, rows, gates=gates, residual=x, stream=stream)
        dr, dg = R.rft_expert_combine_bwd(o, out, rows, gates=gates, stream=stream)
        n = int((ids >= 0).logical_and(ids < E).sum()) if stream is None and not capturing else 0
        return o, out, dg, rows, dr, n

    capturing = False
    first = call()
    n = first[-1]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = call(side)
    torch.cuda.current_stream().wait_stream(side)
    same = lambda a, b: (torch.equal(a[0].slots, b[0].slots) and torch.equal(a[0].places, b[0].places)  # noqa: E731
                         and torch.equal(a[0].offsets, b[0].offsets) and torch.equal(a[1], b[1])
                         and torch.equal(a[2], b[2]) and torch.equal(a[3][:n], b[3][:n])
                         and torch.equal(a[4][:n], b[4][:n]))
    assert same(first, other)
    capturing = True
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    capturing = False
    for _ in range(3):
        held[1].zero_()
        held[0].slots.zero_()
        graph.replay()
        again = call()
        torch.cuda.synchronize()
        assert same(first, held) and same(first, again)


def test_past_32_bits():
    """Rows of more than 2^32 elements: the last tokens' ways to their experts and back."""
    T, E, k, d = 300_000, 16, 8, 2048
    g = torch.Generator(device=DEV).manual_seed(2)
    ids = torch.randint(0, E, (T, k), generator=g, device=DEV, dtype=torch.int32)
    x = torch.randn(T, d, generator=g, device=DEV, dtype=BF)
    gates = torch.rand(T, k, generator=g, device=DEV)
    o = R.rft_expert_sort(ids, E)
    flat = ids.reshape(-1).long()
    order = torch.sort(flat, stable=True)[1]
    assert torch.equal(o.slots.long(), order)
    assert torch.equal(o.places.reshape(-1).long()[order], torch.arange(T * k, device=DEV))
    rows = R.rft_expert_gather(o, x)
    last = torch.tensor([0, 1, T * k // 2, T * k - 2, T * k - 1], device=DEV)
    assert torch.equal(rows[last], x[order[last] // k])
    at = slice(T - 200, T)
    out = R.rft_expert_combine(o, rows, gates=gates)
    want = gates[at].double().sum(1, keepdim=True) * x[at].double()
    tol = (k + 2) * 2.0 ** -24 * want.abs()
    assert bool(((out[at].double() - want).abs() <= tol + torch.finfo(BF).eps / 2 * (want.abs() + tol)).all())
    d_rows, d_gates = R.rft_expert_combine_bwd(o, x, rows, gates=gates, d_rows=rows)
    want = x[at].double().square().sum(1, keepdim=True).expand(200, k)
    assert bool(((d_gates[at].double() - want).abs() <= (d + 2) * 2.0 ** -24 * want).all())
    s = order[last]
    want = gates.reshape(-1)[s, None].double() * x[s // k].double()
    assert bool(((d_rows[last].double() - want).abs() <= (torch.finfo(BF).eps / 2 + 2.0 ** -24) * want.abs()).all())

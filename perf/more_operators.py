"""Operators that take a policy's tokens through the experts that its router chose.

  tokens      rft_expert_sort, rft_expert_gather, rft_expert_combine (and, for training,
              rft_expert_combine_bwd and the gather's gradient): slots sorted by expert, the tokens'
              rows in that order, the experts' rows back with their gates and a residual
  linear      rft_linear: rows of every expert (or of one dense layer) times its weight, with bias,
              activation and residual in the epilogue; the rows may be taken from the tokens' own
              array by the sorted order
  linear_bwd  rft_linear_bwd: gradients to the rows, the weights and the bias

Where `own` is false, run() computes the same in elementary torch operations.
"""
import math

import torch

own = False

DEV = "cuda"
ACTS = ("none", "silu", "gelu", "swiglu")


def _tokens(name, **kw):
    c = dict(name=name, kind="tokens", train=True, dtype="bf16", n_seq=1, lo=1, pad=1, E=64, k=4, d=1536)
    c.update(kw)
    return c


def _linear(name, **kw):
    """rows of tokens * k slots over E experts; E = 1: a dense layer over `tokens` rows."""
    c = dict(name=name, kind="linear", dtype="bf16", tokens=1, k=1, E=1, K=1536, N=1536, act="none",
             bias=False, residual=False, z=False, gather=False)
    c.update(kw)
    return c


def _bwd(name, **kw):
    c = dict(name=name, kind="linear_bwd", dtype="bf16", tokens=1, k=1, E=1, K=1536, N=1536, act="none",
             bias=False, gather=False, dw="bf16")
    c.update(kw)
    return c


def listed():
    return [
        # a decode step over the running sequences of a rollout engine, forward alone
        _tokens("tokens_decode", train=False, n_seq=200, E=256, k=8),
        # a micro-batch of four padded rollouts, fp32 activations, few experts
        _tokens("tokens_micro_f32", dtype="f32", n_seq=4, lo=64, pad=512, E=60, k=4, d=3584),
        # 64 rollouts padded to 1024 rows through 128 experts, forward and backward
        _tokens("tokens_batch", n_seq=64, lo=256, pad=1024, E=128, k=8),
        # one token through the 8 experts it chose, of 128: the smallest call, gate and up projection
        _linear("linear_token", tokens=1, k=8, E=128, act="swiglu", gather=True),
        # a decode step of 200 sequences through 64 experts
        _linear("linear_decode", tokens=200, k=8, E=64, act="swiglu", gather=True),
        # the dense down projection of the 7B-shape policy for 24 sequences, the residual added
        _linear("linear_dense_decode", tokens=24, K=18944, N=3584, residual=True),
        # the experts' gate and up projections of a training micro-batch, z kept for the backward
        _linear("linear_experts", tokens=4096, k=8, E=64, act="swiglu", z=True, gather=True),
        # its backward: to the gathered rows and the experts' weights
        _bwd("bwd_experts", tokens=4096, k=8, E=64, act="swiglu", gather=True),
        # the dense up projection of the 7B-shape policy over a training micro-batch
        _linear("linear_dense", tokens=16384, K=3584, N=18944, act="silu", bias=True, z=True),
        # the gradient of the dense projection without activation, fp32 weight gradients
        _bwd("bwd_dense", tokens=8192, K=3584, N=18944, dw="f32", bias=True),
        # fp32 layers of odd sizes, a few experts
        _linear("linear_odd_f32", dtype="f32", tokens=1111, k=2, E=5, K=1001, N=1537, act="gelu",
                bias=True, residual=True),
        _bwd("bwd_odd_f32", dtype="f32", tokens=777, k=2, E=7, K=515, N=1026, act="swiglu", bias=True,
             dw="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tokens", "linear", "linear", "linear_bwd"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    step = 8 if dtype == "bf16" else 1  # of the sizes
    if kind == "tokens":
        E, d = _log(rng, 4, 512), step * _log(rng, 64 // step, 4096 // step)
        k = min(E, _log(rng, 1, 10))
        train = rng.random() < 0.6
        most = int(8.0e8) // (d * k * (2 if dtype == "bf16" else 4))
        rows = max(1, min(_log(rng, 1, 131072 if train else 4096), most))
        pad = min(rows, _log(rng, 1, 2048)) if train else 1
        c = _tokens("", train=train, dtype=dtype, n_seq=max(1, rows // pad),
                    lo=max(1, pad // rng.choice([1, 2, 8])), pad=pad, E=E, k=k, d=d)
        c.pop("name")
        return c
    K = step * _log(rng, 64 // step, 4096 // step)
    N = step * _log(rng, 64 // step, 8192 // step)
    act = rng.choice(ACTS)
    if act == "swiglu":
        N += N // step % 2 * step  # two halves of whole steps
        N = max(2 * step, N // (2 * step) * 2 * step)
    E = min(rng.choice([1, 1, _log(rng, 2, 160), _log(rng, 2, 160)]), max(1, int(4e8 / (K * N))))
    k = 1 if E == 1 else min(E, rng.randint(1, 8))
    flops = 2.0e12 if dtype == "bf16" else 1.0e11
    most = int(min(flops / (2.0 * K * N * k), 2.0e8 / (max(K, N) * k)))
    tokens = max(1, min(_log(rng, 1, 32768), most))
    if kind == "linear":
        c = _linear("", dtype=dtype, tokens=tokens, k=k, E=E, K=K, N=N, act=act,
                    bias=rng.random() < 0.4, residual=rng.random() < 0.3,
                    z=act != "none" and rng.random() < 0.5, gather=E > 1 and rng.random() < 0.6)
    else:
        dw = "f32" if dtype == "f32" or (act == "none" and rng.random() < 0.5) else "bf16"
        c = _bwd("", dtype=dtype, tokens=max(1, tokens // 2), k=k, E=E, K=K, N=N, act=act,
                 bias=rng.random() < 0.4, gather=E > 1 and rng.random() < 0.6, dw=dw)
    c.pop("name")
    return c


# ---------------------------------------------------------------------------- inputs --
def _dt(s):
    return torch.bfloat16 if s == "bf16" else torch.float32


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _choose(g, T, E, k):
    """A router's choice: a popularity per expert makes the load uneven."""
    z = _randn(g, T, E) + 0.6 * _randn(g, E)
    return torch.topk(z, k, dim=1).indices.int(), torch.softmax(_randn(g, T, k), dim=1)


def prepare(case, seed):
    c, g = dict(case), torch.Generator(device=DEV).manual_seed(int(seed))
    dt = _dt(c["dtype"])
    s = {"c": c}
    if c["kind"] == "tokens":
        T, k, d = c["n_seq"] * c["pad"], c["k"], c["d"]
        n = T * k
        ids, gates = _choose(g, T, c["E"], k)
        if c["pad"] > 1:  # a padded batch: rows past a rollout's length have no expert
            length = torch.randint(c["lo"], c["pad"] + 1, (c["n_seq"],), generator=g, device=DEV)
            live = (torch.arange(c["pad"], device=DEV)[None, :] < length[:, None]).reshape(-1, 1)
            ids = torch.where(live, ids, torch.full_like(ids, -1))
            gates = gates * live
        s.update(ids=ids.contiguous(), gates=gates.contiguous(), x=_randn(g, T, d).to(dt))
        s["residual"] = _randn(g, T, d).to(dt)
        s["y"] = _randn(g, n, d).to(dt)                      # what the experts returned
        s["rows"] = torch.zeros((n, d), dtype=dt, device=DEV)  # rows of no slot stay as they are
        if c["train"]:
            s["d_out"] = _randn(g, T, d).to(dt)
            s["d_rows"] = _randn(g, n, d).to(dt)             # the experts' gradient to their rows
            s["d_y"] = torch.zeros((n, d), dtype=dt, device=DEV)
        return s
    T, k, E, K, N = c["tokens"], c["k"], c["E"], c["K"], c["N"]
    n = T * k
    w = torch.empty((E, N, K), dtype=dt, device=DEV)
    for e in range(E):
        w[e] = _randn(g, N, K) / math.sqrt(K)
    s["w"] = w
    if E > 1:
        ids, _ = _choose(g, T, E, k)
        expert, slots = torch.sort(ids.reshape(-1), stable=True)
        counts = torch.bincount(expert, minlength=E)
        s["expert"], s["slots"] = expert.long(), slots.int()
        s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
        s["cap"] = int(counts.max())
    else:
        s["expert"], s["cap"] = torch.zeros(n, dtype=torch.int64, device=DEV), n
        s["slots"], s["offsets"] = None, None
    s["x"] = _randn(g, T if c["gather"] else n, K).to(dt)
    s["bias"] = (0.1 * _randn(g, E, N)).to(dt) if c["bias"] else None
    M = N // 2 if c["act"] == "swiglu" else N
    if c["kind"] == "linear":
        s["residual"] = _randn(g, n, M).to(dt) if c["residual"] else None
    else:
        s["dy"] = _randn(g, n, M).to(dt)
        s["z"] = _randn(g, n, N).to(dt) if c["act"] != "none" else None
    return s


# ------------------------------------------------------------------- plain operators --
def _plain_tokens(s):
    c = s["c"]
    E, k = c["E"], c["k"]
    ids, dt = s["ids"].reshape(-1).long(), s["x"].dtype
    n, T = ids.numel(), s["ids"].shape[0]
    valid = (ids >= 0) & (ids < E)
    key = torch.where(valid, ids, torch.full_like(ids, E))
    key, order = torch.sort(key, stable=True)
    filled = key < E
    offsets = torch.searchsorted(key, torch.arange(E + 1, device=DEV))
    slots = torch.where(filled, order, torch.full_like(order, -1))
    r = torch.arange(n, device=DEV)
    places = torch.empty_like(r)
    places[order] = torch.where(filled, r, torch.full_like(r, -1))
    token = order // k
    rows = torch.where(filled[:, None], s["x"][token], s["rows"])
    has = (places >= 0)[:, None]
    at = places.clamp(min=0)
    y = torch.where(has, s["y"].float()[at], torch.zeros((), device=DEV))  # in the slots' order
    out = s["residual"].float() + (s["gates"].reshape(-1, 1) * y).view(T, k, -1).sum(1)
    res = {"offsets": offsets.int(), "slots": slots.int(), "places": places.int().view(T, k),
           "rows": rows, "out": out.to(dt)}
    if c["train"]:
        go = s["d_out"].float()
        d_gates = (go[:, None, :] * y.view(T, k, -1)).sum(2)
        weighted = s["gates"].reshape(-1)[order, None] * go[token]
        d_y = torch.where(filled[:, None], weighted.to(dt), s["d_y"])
        back = torch.where(has, s["d_rows"].float()[at], torch.zeros((), device=DEV))
        res.update(d_y=d_y, d_gates=d_gates, d_x=back.view(T, k, -1).sum(1).to(dt))
    return res


def _act(z, act):
    if act == "none":
        return z
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    g, u = z.chunk(2, dim=1)
    return g / (1 + torch.exp(-g)) * u


def _act_bwd(dy, z, act):
    if act == "none":
        return dy
    if act == "gelu":
        return dy * (0.5 * torch.erfc(-z * math.sqrt(0.5))
                     + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi))
    g = z.chunk(2, dim=1)[0] if act == "swiglu" else z
    sig = 1 / (1 + torch.exp(-g))
    slope = sig * (1 + g * (1 - sig))
    if act == "silu":
        return dy * slope
    return torch.cat([dy * z.chunk(2, dim=1)[1] * slope, dy * g * sig], dim=1)


def _inputs(s):
    """The grouped rows of x, in 32 bits."""
    x = s["x"].float()
    return x[s["slots"].long() // s["c"]["k"]] if s["c"]["gather"] else x


def _padded(s, a):
    """Rows [n, C] as [E, cap, C] with zeros behind each expert's rows; and where they went."""
    E, cap = s["c"]["E"], s["cap"]
    r = torch.arange(a.shape[0], device=DEV)
    at = s["expert"] * cap + (r if s["offsets"] is None else r - s["offsets"].long()[s["expert"]])
    p = torch.zeros((E * cap, a.shape[1]), dtype=a.dtype, device=DEV)
    p[at] = a
    return p.view(E, cap, -1), at


def _plain_linear(s):
    c, n = s["c"], s["expert"].numel()
    x = _inputs(s)
    if c["E"] > 1 and n <= 64:  # a few rows: each with the weight of its own expert
        z = (s["w"][s["expert"]].float() * x[:, None, :]).sum(2)
    else:
        p, at = _padded(s, x)
        z = torch.matmul(p, s["w"].float().transpose(1, 2).contiguous()).flatten(0, 1)[at]
    if s["bias"] is not None:
        z = z + s["bias"].float()[s["expert"]]
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    dt = s["x"].dtype
    return {"y": y.to(dt), "z": z.to(dt)} if c["z"] else {"y": y.to(dt)}


def _plain_bwd(s):
    c, dt = s["c"], s["x"].dtype
    dz = _act_bwd(s["dy"].float(), None if s["z"] is None else s["z"].float(), c["act"])
    p, at = _padded(s, dz)
    q, _ = _padded(s, _inputs(s))
    res = {"d_x": torch.matmul(p, s["w"].float()).flatten(0, 1)[at].to(dt),
           "d_w": torch.matmul(p.transpose(1, 2).contiguous(), q).to(_dt(c["dw"]))}
    if c["bias"]:
        res["d_b"] = p.double().sum(1).float()
    return res


# --------------------------------------------------------------- the package's calls --
def _own(s):
    import paper_2505_17826_amd as R
    c = s["c"]
    if c["kind"] == "tokens":
        o = R.rft_expert_sort(s["ids"], c["E"])
        rows = R.rft_expert_gather(o, s["x"], out=s["rows"])
        out = R.rft_expert_combine(o, s["y"], gates=s["gates"], residual=s["residual"])
        res = {"offsets": o.offsets, "slots": o.slots, "places": o.places, "rows": rows, "out": out}
        if c["train"]:
            d_y, d_gates = R.rft_expert_combine_bwd(o, s["d_out"], s["y"], gates=s["gates"],
                                                    d_rows=s["d_y"])
            res.update(d_y=d_y, d_gates=d_gates, d_x=R.rft_expert_combine(o, s["d_rows"]))
        return res
    groups = None
    if c["E"] > 1:
        groups = R.Groups(s["offsets"], s["slots"] if c["gather"] else None, c["k"])
    act = (R.RFT_ACT_NONE, R.RFT_ACT_SILU, R.RFT_ACT_GELU, R.RFT_ACT_SWIGLU)[ACTS.index(c["act"])]
    if c["kind"] == "linear":
        y, z = R.rft_linear(s["x"], s["w"], bias=s["bias"], act=act, residual=s["residual"],
                            groups=groups, want_z=c["z"])
        return {"y": y, "z": z} if c["z"] else {"y": y}
    d_x, d_w, d_b = R.rft_linear_bwd(s["dy"], s["x"], s["w"], z=s["z"], act=act, groups=groups,
                                     dw_dtype=_dt(c["dw"]), want_db=c["bias"])
    return {"d_x": d_x, "d_w": d_w, "d_b": d_b} if c["bias"] else {"d_x": d_x, "d_w": d_w}


def run(state):
    if own:
        return _own(state)
    kind = state["c"]["kind"]
    return (_plain_tokens if kind == "tokens" else _plain_linear if kind == "linear" else _plain_bwd)(state)


# ------------------------------------------------------------------- 64-bit results --
def _exact_tokens(s):
    c = s["c"]
    T, k = s["ids"].shape
    ids = s["ids"].cpu()
    # by the definition: expert after expert, its slots in ascending order
    order = torch.cat([(ids.reshape(-1) == e).nonzero()[:, 0] for e in range(c["E"])]).to(DEV)
    n = order.numel()
    rows = s["rows"].double()
    rows[:n] = s["x"].double()[order // k]
    gate = s["gates"].double().reshape(-1)[order]
    out = s["residual"].double()
    out.index_add_(0, order // k, gate[:, None] * s["y"][:n].double())
    res = {"offsets": None, "slots": None, "places": None, "rows": rows, "out": out}
    if c["train"]:
        go = s["d_out"].double()[order // k]
        d_y = s["d_y"].double()
        d_y[:n] = gate[:, None] * go
        d_gates = torch.zeros(T * k, dtype=torch.float64, device=DEV)
        d_gates[order] = (go * s["y"][:n].double()).sum(1)
        d_x = torch.zeros(s["x"].shape, dtype=torch.float64, device=DEV)
        d_x.index_add_(0, order // k, s["d_rows"][:n].double())
        res.update(d_y=d_y, d_gates=d_gates.view(T, k), d_x=d_x)
    return res


def _value(z, act):
    """act of z and its slopes by autograd's definition, written out: (value, slope factors)."""
    if act == "none":
        return z, (torch.ones_like(z),)
    if act == "gelu":
        cdf = 0.5 * (1 + torch.erf(z / math.sqrt(2.0)))
        return z * cdf, (cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),)
    g = z[:, :z.shape[1] // 2] if act == "swiglu" else z
    sig = torch.sigmoid(g)
    silu, slope = g * sig, sig + g * sig * (1 - sig)
    if act == "silu":
        return silu, (slope,)
    u = z[:, z.shape[1] // 2:]
    return silu * u, (u * slope, silu)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] == "tokens":
        return _exact_tokens(s)
    n = s["expert"].numel()
    start = [0, n] if s["offsets"] is None else s["offsets"].tolist()
    forward = c["kind"] == "linear"
    keep = {q: [] for q in ("y", "z", "d_x")}
    d_w, d_b = torch.zeros(0), torch.zeros(0)
    if not forward:
        d_w = torch.zeros(s["w"].shape, dtype=torch.float64, device=DEV)
        d_b = torch.zeros((c["E"], c["N"]), dtype=torch.float64, device=DEV)
    for e in range(c["E"]):
        a, b = start[e], start[e + 1]
        if a == b:
            continue
        x = s["x"][s["slots"][a:b].long() // c["k"]].double() if c["gather"] else s["x"][a:b].double()
        w = s["w"][e].double()
        if forward:
            z = x @ w.t().contiguous()
            if c["bias"]:
                z = z + s["bias"][e].double()
            y, _ = _value(z, c["act"])
            keep["y"].append(y + s["residual"][a:b].double() if c["residual"] else y)
            keep["z"].append(z if c["z"] else z[:0])
        else:
            dy = s["dy"][a:b].double()
            slopes = _value(s["z"][a:b].double(), c["act"])[1] if s["z"] is not None else (1.0,)
            dz = torch.cat([dy * q for q in slopes], dim=1)
            keep["d_x"].append(dz @ w)
            d_w[e] = dz.t().contiguous() @ x
            d_b[e] = dz.sum(0)
    if forward:
        res = {"y": torch.cat(keep["y"])}
        return dict(res, z=torch.cat(keep["z"])) if c["z"] else res
    res = {"d_x": torch.cat(keep["d_x"]), "d_w": d_w}
    return dict(res, d_b=d_b) if c["bias"] else res


# -------------------------------------------------------------------------- the work --
def work(case):
    c = case
    w = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "tokens":
        T, k = c["n_seq"] * c["pad"], c["k"]
        live = c["n_seq"] * (c["lo"] + c["pad"]) / 2 if c["pad"] > 1 else T  # tokens with experts
        n = live * k
        row = c["d"] * w
        b = 4 * T * k + 8 * T * k + 4 * T * k           # ids in, the order out, gates in
        b += (live + n) * row + (n + 2 * T) * row       # gather; combine with the residual
        fl = 2 * n * c["d"]
        if c["train"]:
            b += (live + 2 * n) * row + 8 * T * k       # gradients to the experts' rows and the gates
            b += (n + T) * row                          # and of the gather
            fl += 4 * n * c["d"]
        return {"bytes": b, "flops": fl}
    n, K, N, E = c["tokens"] * c["k"], c["K"], c["N"], c["E"]
    M = N // 2 if c["act"] == "swiglu" else N
    used = min(E, n) if n < 4 * E else E                # experts with rows, about
    x = c["tokens"] if c["gather"] else n
    if c["kind"] == "linear":
        b = w * (x * K + used * N * K + n * M * (2 if c["residual"] else 1) + (n * N if c["z"] else 0))
        return {"bytes": b, "flops": 2 * n * N * K}
    b = w * (x * K + used * N * K + n * M + n * K + (n * N if c["act"] != "none" else 0))
    b += E * N * K * (2 if c["dw"] == "bf16" else 4)
    return {"bytes": b, "flops": 4 * n * N * K}

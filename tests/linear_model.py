"""Linear layers over groups of rows in plain float64 (CPU): values, gradients and the scales
that the roundings of the kernels are measured by."""
import math

import torch

ACTS = ("none", "silu", "gelu", "swiglu")


def value(z, act):
    if act == "none":
        return z
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    g = z[:, :z.shape[1] // 2] if act == "swiglu" else z
    s = g * torch.sigmoid(g)
    s = torch.where(g == -math.inf, torch.zeros_like(s), s)
    return s * z[:, z.shape[1] // 2:] if act == "swiglu" else s


def slopes(z, act):
    """d value / d z, per half for swiglu."""
    if act == "none":
        return (torch.ones_like(z),)
    if act == "gelu":
        return (0.5 * torch.erfc(-z / math.sqrt(2))
                + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),)
    g = z[:, :z.shape[1] // 2] if act == "swiglu" else z
    s = torch.sigmoid(g)
    d = s * (1 + g * (1 - s))
    if act == "silu":
        return (d,)
    return (z[:, z.shape[1] // 2:] * d, g * s)


def rows_of_x(x, source, div, rows):
    if source is None:
        return x[:rows]
    t = torch.div(source.long(), div, rounding_mode="floor")
    ok = (source >= 0) & (t < x.shape[0])
    out = x.new_zeros(rows, x.shape[1])
    out[ok] = x[t[ok]]
    return out


def forward(x, w, bias, act, residual, offsets, rows_x=None):
    """float64; rows of no group are NaN.  Returns y, z and the sums of magnitudes behind z."""
    E, n, _ = w.shape
    rows = x.shape[0]
    z = torch.full((rows, n), math.nan, dtype=torch.float64)
    mag = torch.zeros_like(z)
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        z[a:b] = x[a:b] @ w[e].T
        mag[a:b] = x[a:b].abs() @ w[e].abs().T
        if bias is not None:
            z[a:b] += bias[e]
            mag[a:b] += bias[e].abs()
    y = value(z, act)
    if residual is not None:
        y = y + residual
    return y, z, mag


def backward(dy, z, x, w, act, offsets):
    """d_x, d_w, d_b, dz and the sums of magnitudes behind d_x, d_w, d_b."""
    E, n, k = w.shape
    rows = x.shape[0]
    dz = torch.full((rows, n), math.nan, dtype=torch.float64)
    dx = torch.full((rows, k), math.nan, dtype=torch.float64)
    dw, db = torch.zeros(E, n, k, dtype=torch.float64), torch.zeros(E, n, dtype=torch.float64)
    mx, mw, mb = torch.zeros_like(dx), torch.zeros_like(dw), torch.zeros_like(db)
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        s = slopes(z[a:b], act) if act != "none" else (1.0,)
        dz[a:b] = torch.cat([dy[a:b] * q for q in s], 1)
        dx[a:b], mx[a:b] = dz[a:b] @ w[e], dz[a:b].abs() @ w[e].abs()
        dw[e], mw[e] = dz[a:b].T @ x[a:b], dz[a:b].abs().T @ x[a:b].abs()
        db[e], mb[e] = dz[a:b].sum(0), dz[a:b].abs().sum(0)
    return dx, dw, db, dz, mx, mw, mb

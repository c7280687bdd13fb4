"""The arithmetic of the orthogonalisation on the host: the iteration in float64 with every
rounding of an operand to fp16 (or to a sum of two) made where the kernels make it, and the
limits that the documented errors set.  Sums are exact here, fp32 in the kernels."""
import math

import torch

COEFS = (3.4445, -4.7750, 2.0315)
# documented for RFT_PRODUCTS_ONE: errors of about 1e-3, below those of a bf16 result (1.65e-3)
ONE = 1e-3


def three(g):
    """RFT_PRODUCTS_THREE, errors as of fp32 products: twice those of the iteration in fp32 here,
    and where that is nearly exact a few roundings to 22 bits."""
    return 2 * error(iterate(g.float()), g) + 4 * 2.0 ** -22


def gradient(seed, *shape):
    """Noise and a few strong directions, as a gradient has."""
    g = torch.Generator().manual_seed(seed)
    m, n = shape[-2:]
    r = min(4, m, n)
    s = 4 * (math.sqrt(m) + math.sqrt(n)) / math.sqrt(m * n)
    u = torch.randn(*shape[:-1], r, generator=g)
    v = torch.randn(*shape[:-2], r, n, generator=g)
    return torch.randn(*shape, generator=g) + s * u @ v


def _short_side(f):
    def call(g, *a, **k):
        if g.shape[-2] > g.shape[-1]:
            return f(g.transpose(-1, -2), *a, **k).transpose(-1, -2)
        return f(g, *a, **k)
    return call


@_short_side
def iterate(g, steps=5):
    """In g's own type."""
    a, b, c = COEFS
    x = g / torch.linalg.matrix_norm(g, keepdim=True)
    for _ in range(steps):
        y = x @ x.transpose(-1, -2).contiguous()
        x = a * x + (b * y + c * y @ y) @ x
    return x


def error(x, g):
    """Relative, in the 2-norm of the result; the worst of a stack."""
    ref = iterate(g.double())
    d = (x.double() - ref).flatten(-2).norm(dim=-1)
    return float((d / ref.flatten(-2).norm(dim=-1)).max())


def _hi(x):
    return (x * 4096).half().double() / 4096


def _pair(x):
    h = _hi(x)
    return h + _hi(x - h)


@_short_side
def model(g, products=1, diagonals_rounded=False):
    """One matrix.  diagonals_rounded: a mistake, the diagonals of A and of its polynomial in the
    fp16 operands instead of apart in fp32."""
    a, b, c = COEFS

    def mul(x, y):
        r = _hi(x) @ _hi(y)
        return r if products == 1 else r + _hi(x) @ _hi(y - _hi(y)) + _hi(x - _hi(x)) @ _hi(y)

    held = _hi if products == 1 else _pair
    x = _pair(g.double() / g.double().norm())
    for i in range(5):
        A = mul(x, x.T)
        d = A.diagonal().clone()
        if diagonals_rounded:
            o = held(A)
            x = a * x + mul(held(b * o + c * mul(o, o)), x)
        else:
            o = held(A - torch.diag(d))
            s = mul(o, o)
            p = a + b * d + c * (s.diagonal() + d * d)
            P = b * o + c * (s + (d[:, None] + d[None]) * o)
            x = p[:, None] * x + mul(held(P - torch.diag(P.diagonal())), x)
        x = _pair(x) if i < 4 else x
    return x

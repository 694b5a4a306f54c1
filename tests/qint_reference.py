"""Plain 64-bit definitions of the operators on 8-bit integers, for the tests: written from the
format's definition (include/dlm.h), sharing no code with the library."""
import math

import torch

ROW, MAX_K = 128, 131071
U = 2.0 ** -24                 # half a step of fp32, relative
NEAR = 2.0 ** -40              # of a step: how near the middle either neighbour will do


def row_bytes(k):
    return -(-k // ROW) * ROW


def check_packed(codes, scales, x, like=None):
    """codes [n, K] and scales [n] (CPU) are a packing of x [n, k] (64 bits): every code is an
    integer nearest to x min(127 / A, 2^126), every scale the fp32 number nearest to max(A / 127,
    2^-126) (off by half a step, and what the 64-bit arithmetic before it may move: 2^-40)."""
    n, k = x.shape
    assert codes.shape == (n, row_bytes(k)) and codes.dtype == torch.int8
    assert not codes[:, k:].any(), "codes behind k"
    bad = ~torch.isfinite(x).all(1)
    assert bool(scales[bad].isnan().all()) and not codes[bad].any()
    x, c, s = x[~bad], codes[~bad, :k].double(), scales[~bad].double()
    a = x.abs().amax(1)
    want = (a / 127).clamp_min(2.0 ** -126)
    assert bool(((s - want).abs() <= want * (U + NEAR)).all())
    v = x * torch.where(a > 0, 127 / a.clamp_min(1e-300), torch.full_like(a, math.inf)).clamp_max(2.0 ** 126)[:, None]
    off = (c - v).abs()
    assert bool((off <= 0.5 + NEAR).all()), float(off.max())
    if like is not None:       # rows whose step is a power of two: ties go to the even code
        assert torch.equal(c[like], torch.round(v[like]))


def pack(x):
    """codes and scales of x [n, k] (CPU), by the definition."""
    n, k = x.shape
    x = x.double()
    bad = ~torch.isfinite(x).all(1)
    y = torch.where(bad[:, None], torch.zeros_like(x), x)
    a = y.abs().amax(1)
    r = torch.where(a > 0, 127 / a.clamp_min(1e-300), torch.full_like(a, math.inf)).clamp_max(2.0 ** 126)
    codes = torch.zeros(n, row_bytes(k), dtype=torch.int8)
    codes[:, :k] = torch.round(y * r[:, None]).to(torch.int8)
    scales = (a / 127).clamp_min(2.0 ** -126).float()
    return codes, torch.where(bad, torch.full_like(scales, math.nan), scales)


def half_ulp(x, dtype):
    """Half a step of the type at |x|."""
    a = x.abs().clamp_min(2.0 ** -126)
    return 2.0 ** (torch.floor(torch.log2(a)) - (8 if dtype == torch.bfloat16 else 24))


def product(xc, xs, wc, ws):
    """(p, bound) in 64 bits: the sums are exact there; their conversion and two scalings are off
    by half a step each, (1 + u)^3 - 1 < 3.001 u."""
    acc = xc.double() @ wc.double().T              # whole numbers below 2^53
    p = acc * xs.double()[:, None] * ws.double()[None]
    return p, 3.001 * U * p.abs()


def silu_mul(g, u):
    return g * torch.sigmoid(g) * u


def swiglu(p, bound):
    """(y, bound) of gate and up halves: the products' bounds through silu(g) u (|silu'| <= 1.1,
    |silu(g)| <= |g|), and of the fp32 steps: the exponential's argument |g| u, itself and the sum,
    the quotient and the product 8 u. Below -87.3 the quotient is a subnormal number or the
    exponential overflows, and silu may become zero: it is less than 2^-119 there."""
    g, u = p.chunk(2, 1)
    tg, tu = bound.chunk(2, 1)
    y = silu_mul(g, u)
    return y, (1.1 * tg * (u.abs() + tu) + g.abs() * tu + (g.abs() + 8) * U * y.abs() +
               2.0 ** -119 * (u.abs() + tu))

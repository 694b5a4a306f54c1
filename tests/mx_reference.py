"""Plain 64-bit definitions of the 4-bit operators, for the tests: written from the
format's definition (include/dlm.h), sharing no code with the library."""
import math

import torch

GROUP = 32
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
U = 2.0 ** -24


def groups(k):
    return -(-k // GROUP)


def scale_stride(k):
    return -(-groups(k) // 16) * 16


def pack(w):
    """codes [n, 16 G] and scales [n, S] of w [n, k] (a CPU tensor)."""
    n, k = w.shape
    x = torch.zeros(n, groups(k) * GROUP, dtype=torch.float64)
    x[:, :k] = w.double()
    x = x.reshape(n, groups(k), GROUP)
    bad = ~torch.isfinite(x).all(-1)
    x = torch.where(bad[..., None], torch.zeros_like(x), x)
    amax = x.abs().amax(-1)
    e = torch.ceil(torch.log2((amax / 7).clamp_min(2.0 ** -1000)))
    # (log2 of a value next to a power of two: settle the border exactly)
    e = torch.where(amax > 7 * 2.0 ** e, e + 1, torch.where(amax <= 7 * 2.0 ** (e - 1), e - 1, e))
    e = e.clamp(-125, 125)
    y = x.abs() / (2.0 ** e)[..., None]
    levels = torch.tensor(LEVELS, dtype=torch.float64)
    d = (y[..., None] - levels).abs()
    # nearest level; of two equally near ones the even code
    d = d + 1e-9 * (torch.arange(8) % 2) * (d == d.amin(-1, keepdim=True))
    code = d.argmin(-1) + 8 * torch.signbit(x).long()
    code = torch.where(bad[..., None], torch.zeros_like(code), code).reshape(n, groups(k) * GROUP)
    codes = (code[:, 0::2] + 16 * code[:, 1::2]).to(torch.uint8)
    scales = torch.zeros(n, scale_stride(k), dtype=torch.uint8)
    scales[:, :groups(k)] = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return codes, scales


def values(codes, scales, k):
    """The values [n, k] in 64 bits."""
    c = codes.long().cpu()
    nib = torch.stack([c % 16, c // 16], -1).flatten(1)
    mag = torch.tensor(LEVELS, dtype=torch.float64)[nib % 8]
    e = scales[:, :groups(k)].cpu().double().repeat_interleave(GROUP, 1)
    v = torch.where(nib >= 8, -mag, mag) * 2.0 ** (e - 127)
    return torch.where(e == 255, torch.full_like(v, math.nan), v)[:, :k]


def half_ulp(x, dtype):
    """Half a step of the type at |x|."""
    a = x.abs().clamp_min(2.0 ** -126)
    return 2.0 ** (torch.floor(torch.log2(a)) - (8 if dtype == torch.bfloat16 else 24))


def product_bound(x, w, dtype):
    """What fp32 accumulation may be off by: every 32-wide MFMA step adds to an fp32 sum,
    the waves' parts are added at the end (at most 16); fp32 inputs enter as
    three terms, each a step, the last one rounded to 2^-25 of the input."""
    k = x.shape[1]
    steps = k / 32 + 4 if dtype == torch.bfloat16 else 3 * (k / 32 + 4) + 1
    return (steps + 18) * U * (x.abs() @ w.abs().T)


def silu_mul(g, u):
    return g / (1 + torch.exp(-g)) * u


def swiglu_bound(g, u, tg, tu, dtype):
    """The products' bounds through silu(g) u (|silu'| <= 1.1, |silu(g)| <= |g|), 8 u for the
    exponential, the division and the product, and the rounding to the type."""
    y = silu_mul(g, u)
    return 1.1 * tg * (u.abs() + tu) + g.abs() * tu + 8 * U * y.abs() + half_ulp(y, dtype)


def rotate32(x, rot):
    """fp32 rotation of [N, heads, dh], each operation rounded by itself."""
    a, b = x.chunk(2, -1)
    c, s = rot[:, None, :, 0], rot[:, None, :, 1]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def attention(q, k, v, dtype):
    """(output, bound) of q [n, hq, dh] over k, v [len, hkv, dh], all 64 bits. The bound: a
    weight is off by the fp32 error of its score (dh / 32 + 6 roundings of the dot product's
    terms, and the scaled difference), its exponential (8 u) and, in bf16 models, its
    rounding (2^-9); the sums over the keys by one rounding for each 32. A weight below 2^-126
    of the largest one counts as zero (the exponential has no subnormal results), which
    takes less than 2^-126 |v| from the output for each key."""
    n, hq, dh = q.shape
    L, hkv = k.shape[0], k.shape[1]
    if L == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    gh = hq // hkv
    qh = q.reshape(n, hkv, gh, dh).permute(1, 2, 0, 3).reshape(hkv, gh * n, dh)
    kh, vh = k.permute(1, 0, 2), v.permute(1, 0, 2)
    z = qh @ kh.transpose(1, 2) / math.sqrt(dh)
    p = torch.softmax(z, -1)
    za = (qh.abs() @ kh.abs().transpose(1, 2)).amax(-1, keepdim=True) / math.sqrt(dh)
    planes = 1 if dtype == torch.bfloat16 else 3
    rel = (planes * (dh / 32) + 12) * U * za * 2 + 8 * U + (planes * L / 32 + 24) * U
    rel = rel + (2.0 ** -9 if dtype == torch.bfloat16 else 2.0 ** -24)
    o = p @ vh
    # numerator and denominator are each off by rel
    bound = rel * (p @ vh.abs()) + rel * o.abs() + 2.0 ** -126 * vh.abs().sum(1, keepdim=True)
    back = lambda t: t.reshape(hkv, gh, n, dh).permute(2, 0, 1, 3).reshape(n, hq, dh)
    o, bound = back(o), back(bound)
    return o, bound + half_ulp(o, dtype)

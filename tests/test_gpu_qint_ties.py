"""Codes next to the middle of two, against whole-number arithmetic: rows whose quotients
127 x / A are exact middles go to the even code, whatever A is."""
import pytest
import torch

import qint_reference as ref
from paper_2606_29094_amd import dlm
from test_gpu_qint import _empty, _held

BF16, F32 = torch.bfloat16, torch.float32


def _codes(x):
    """Codes of the rows of x, whole numbers of any common unit (below 2^40), exactly."""
    a = x.abs().amax(1, keepdim=True)
    top = 254 * x.abs() + a                                     # 2 A (q + 1/2)
    c = top // (2 * a)
    c = c - ((top % (2 * a) == 0) & (c % 2 == 1)).long()        # a middle: the even code
    return torch.where(x < 0, -c, c)


def _middles(kind):
    """Rows of whole numbers, each with both signs of every value; their type and unit."""
    if kind == "bf16":             # every significand of A against every one of x, down to A 2^-12
        a = torch.arange(128, 256)[:, None]
        x = torch.cat([torch.arange(128, 256) << e for e in range(13)])[None].repeat(128, 1)
        x = torch.where(x <= a << 12, x, torch.zeros_like(x))
        x[:, 0] = a[:, 0] << 12
    elif kind == "halves":         # A any fp32 number, x = A / 2
        a = torch.randint(1 << 23, 1 << 24, (64, 1), generator=torch.Generator().manual_seed(1))
        x = torch.cat([2 * a, a, torch.zeros_like(a)], 1).repeat(1, 100)
    else:                          # A = 127 m, x = (c + 1/2) m and its neighbours, c = 0 .. 126
        m = torch.cat([torch.arange(1, 33), 2 * torch.randint(16513, 33026, (32,), generator=torch.Generator().manual_seed(2)) + 1])
        mid = (2 * torch.arange(127) + 1)[None] * m[:, None]
        x = torch.cat([254 * m[:, None], mid, mid + 1, mid - 1], 1)
    return torch.cat([x, -x], 1)


def test_reference_is_exact():
    from fractions import Fraction
    for kind in ("bf16", "halves", "127 m"):
        x = _middles(kind)
        c = _codes(x)
        for row in (0, 5, len(x) - 1):
            a = int(x[row].abs().max())
            for i in range(0, x.shape[1], 7):
                assert int(c[row, i]) == round(Fraction(127 * int(x[row, i]), a))     # (ties to even)


def _check(q, x, k):
    codes, scales = _held(q)
    want = torch.zeros(len(x), ref.row_bytes(k), dtype=torch.int8)
    want[:, :k] = _codes(x).to(torch.int8)
    assert torch.equal(codes, want), int((codes != want).sum())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [(BF16, "bf16"), (F32, "bf16"), (F32, "halves"), (F32, "127 m")])
@pytest.mark.parametrize("exponent", [-120, -30, 0, 90])
@pytest.mark.parametrize("times,pad", [(1, 0), (1, 3), (29, 0), (29, 1)])
def test_packed(gpu, dtype, kind, exponent, times, pad):
    """Rows of one pass and of two (29 times as long), whole vectors and others."""
    x = _middles(kind).repeat(1, times)[:8 if times > 1 else None]
    k = x.shape[1]
    v = (x.double() * 2.0 ** exponent).to(dtype)
    assert torch.equal(v.double(), x.double() * 2.0 ** exponent)
    big = torch.zeros(len(x), k + pad, dtype=dtype, device=gpu)
    big[:, :k] = v.to(gpu)
    q = _empty(gpu, len(x), k)
    dlm.qint_pack(big[:, :k], q)
    _check(q, x, k)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "halves", "127 m"])
@pytest.mark.parametrize("times,pad", [(1, 0), (1, 3), (29, 0)])
def test_normed(gpu, kind, times, pad):
    """The norm's codes follow from h' gain; gains that are powers of two keep the middles."""
    x = _middles(kind).repeat(1, times)[:8 if times > 1 else None]
    k = x.shape[1]
    g = 2.0 ** (torch.arange(k) % 5 - 2)
    h = torch.zeros(len(x), k + pad, device=gpu)
    h[:, :k] = (x.double() * 2.0 ** -20 / g).float().to(gpu)
    q = _empty(gpu, len(x), k)
    dlm.qint_norm(h[:, :k], g.to(gpu), 1e-5, q)
    _check(q, x, k)

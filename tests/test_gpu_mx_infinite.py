"""Products with 4-bit matrices whose scales reach beyond bf16 (scale bytes 253 and 254, where
the larger codes stand for infinities)."""
import pytest
import torch

import mx_reference as ref
from paper_2606_29094_amd import dlm
from test_gpu_mx import _randn

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _linear(gpu, x, codes, scales, n, k):
    q = dlm.make_mx(codes.to(gpu), scales.to(gpu), n, k)
    y = torch.empty(x.shape[0], n, device=gpu)
    ws = torch.empty(max(256, dlm.mx_linear_workspace(x.dtype, x.shape[0], q)), dtype=torch.uint8, device=gpu)
    dlm.mx_linear(x.to(gpu), q, y, workspace=ws)
    return y.cpu().double()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m,n,k", [(3, 48, 33), (3, 48, 40), (16, 96, 1031), (20, 48, 520), (70, 48, 8),
                                   (300, 96, 200), (300, 96, 481), (70, 2048, 4072), (600, 4096, 520)])
def test_linear_ignores_infinite_codes_behind_k(gpu, m, n, k, dtype):
    """Codes behind k stand for infinities under the last group's scale, the codes within k for
    finite values: the product is finite."""
    codes, scales = ref.pack(_randn(n, k, seed=k))
    at = (k - 1) // 32                                     # the last group
    inside = torch.randint(0, 3, (n, k - 32 * at), generator=torch.Generator().manual_seed(1))
    nib = torch.full((n, 32), 7)                           # 6 x scale: infinite from byte 253 on
    nib[:, 1::3] = 15
    nib[:, :k - 32 * at] = inside + 8 * (inside % 2)       # 0, -0.5 or 1 scales
    codes[:, 16 * at:] = (nib[:, 0::2] + 16 * nib[:, 1::2]).to(torch.uint8)
    scales[:, at] = torch.where(torch.arange(n) % 3 == 0, 254, 253).to(torch.uint8)
    w = ref.values(codes, scales, k)
    assert w.abs().max() < 2.0 ** 128
    x = _randn(m, k, seed=2, std=2.0 ** -60).to(dtype)     # (the products stay within fp32)
    got, xx = _linear(gpu, x, codes, scales, n, k), x.double()
    assert bool(got.isfinite().all())
    assert bool(((got - xx @ w.T).abs() <= ref.product_bound(xx, w, dtype)).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m,n,k", [(1, 48, 64), (5, 48, 512), (16, 96, 1024), (33, 96, 64), (70, 2048, 4096),
                                   (300, 96, 224), (600, 4096, 512)])
def test_linear_infinite_weights(gpu, m, n, k, dtype):
    """An infinite weight makes its column's outputs infinite, of the sign of its input, whatever
    the input's type; other weights of the same groups stay what they are."""
    codes, scales = ref.pack(_randn(n, k, seed=k))
    at = torch.arange(n) % (k // 32)                       # of each row, one group
    nib = torch.randint(0, 3, (n, 32), generator=torch.Generator().manual_seed(1))
    odd = torch.arange(n) % 2 == 1                         # of each second row, one code
    which = torch.arange(n) * 7 % 32
    nib[odd, which[odd]] = (6 + 8 * (torch.arange(n) // 2 % 2))[odd]
    nib[torch.arange(n) % 8 == 3, 0] = 12 + torch.arange(n)[torch.arange(n) % 8 == 3] // 8 % 4
    packed = (nib[:, 0::2] + 16 * nib[:, 1::2]).to(torch.uint8)
    for r in range(n):
        codes[r, 16 * at[r]:16 * at[r] + 16] = packed[r]
        scales[r, at[r]] = 253 + r // 4 % 2
    w = ref.values(codes, scales, k)
    w = torch.where(w.abs() >= 2.0 ** 128, torch.sign(w) * float("inf"), w)
    x = _randn(m, k, seed=2, std=2.0 ** -60).to(dtype)
    got, xx = _linear(gpu, x, codes, scales, n, k), x.double()
    want = torch.empty(m, n, dtype=torch.float64)
    for r in range(n):                                     # (several infinities: inf or NaN)
        want[:, r] = (xx * w[r]).sum(1)
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
    assert torch.equal(torch.sign(got)[want.isinf()], torch.sign(want)[want.isinf()])
    fin = want.isfinite()
    assert fin.any() and want.isinf().any()
    bound = ref.product_bound(xx, torch.where(w.isfinite(), w, torch.zeros_like(w)), dtype)
    assert bool(((got - want).abs() <= bound)[fin].all())

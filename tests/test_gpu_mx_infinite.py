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

"""Products with 4-bit matrices from 2048 rows on whose operands lie more than 2^32 elements
apart: rows of x far from each other, and a matrix of more than 2^32 values."""
import pytest
import torch

import mx_reference as ref
from paper_2606_29094_amd import dlm
from test_gpu_mx import _randn

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_linear_rows_far_apart(gpu):
    m, n, k, ld = 2050, 1040, 1024, (1 << 21) + 8          # the last row 2^32 elements behind the first
    codes, scales = ref.pack(_randn(n, k, seed=1))
    w = ref.values(codes, scales, k)
    q = dlm.make_mx(codes.to(gpu), scales.to(gpu), n, k)
    x = _randn(m, k, seed=2, dtype=BF16)
    wide = torch.empty(m, ld, dtype=BF16, device=gpu)[:, :k]
    wide.copy_(x)
    y = torch.empty(m, n, device=gpu)
    ws = torch.empty(max(256, dlm.mx_linear_workspace(BF16, m, q)), dtype=torch.uint8, device=gpu)
    dlm.mx_linear(wide, q, y, workspace=ws)
    xx = x.double()
    assert bool(((y.cpu().double() - xx @ w.T).abs() <= ref.product_bound(xx, w, BF16)).all())


def test_linear_matrix_of_more_than_32_bits(gpu):
    m, n, k, period = 2048, 131136, 32768, 64              # n k = 1.0005 x 2^32; rows repeat
    codes, scales = ref.pack(_randn(period, k, seed=1))
    w = ref.values(codes, scales, k)
    q = dlm.make_mx(codes.to(gpu).repeat(n // period, 1), scales.to(gpu).repeat(n // period, 1), n, k)
    x = _randn(m, k, seed=2, dtype=BF16)
    y = torch.empty(m, n, device=gpu)
    ws = torch.empty(max(256, dlm.mx_linear_workspace(BF16, m, q)), dtype=torch.uint8, device=gpu)
    dlm.mx_linear(x.to(gpu), q, y, workspace=ws)
    xx = x.to(gpu).double()
    want = (xx @ w.to(gpu).T.contiguous())
    bound = ref.product_bound(xx, w.to(gpu), BF16)
    for i in range(0, n, period):
        assert bool(((y[:, i:i + period].double() - want).abs() <= bound).all()), i

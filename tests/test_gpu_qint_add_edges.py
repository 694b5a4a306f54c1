"""Sums with a residual in place where the last tiles reach beyond the matrix, scales at a
float's alignment: the places beyond take part in nothing."""
import pytest
import torch

import qint_reference as ref
from paper_2606_29094_amd import dlm
from test_gpu_qint import _check_linear, _randn

pytestmark = pytest.mark.gpu


def _odd_scales(gpu, n, k, seed):
    codes, scales = ref.pack(_randn(n, k, seed=seed))
    held = torch.full((n + 2,), float("nan"), device=gpu)      # (what a scale's neighbours hold)
    held[1:-1] = scales.to(gpu)
    return dlm.make_qint(codes.to(gpu), held[1:-1], n, k), codes[:, :k], scales


# tiles of 256 x 256, 256 x 128 and 256 x 224 with and without sub-tiles, the few-row ones, odd columns
@pytest.mark.parametrize("m,n,k", [(1, 4, 130), (17, 4, 640), (70, 68, 700), (137, 692, 1031), (333, 260, 200),
                                   (600, 3076, 130), (1197, 1644, 1938), (4099, 644, 300), (4099, 645, 300),
                                   (4097, 3588, 260), (8193, 1028, 140)])
def test_residual_in_place(gpu, m, n, k):
    x, w = _odd_scales(gpu, m, k, 1), _odd_scales(gpu, n, k, 2)
    for pad in (0, 4):
        _check_linear(gpu, m, n, k, "add", pad=pad, seed=m, x=x, w=w, in_place=True)

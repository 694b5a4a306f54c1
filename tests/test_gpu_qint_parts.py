"""Products of more rows than the tiles' 32-bit offsets reach, a last part of one row: every
part is computed, the residual is added once."""
import pytest
import torch

import qint_reference as ref
from paper_2606_29094_amd import dlm
from test_gpu_qint import BF16, F32, _matrix, _randn
from test_qint_parts_host import part_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k,epilogue,dtype", [
    (349441, 4, 24576, "store", F32), (349441, 4, 24576, "add", F32), (349441, 4, 24576, "swiglu", BF16),
    (65281, 600, 131071, "add", F32)])
def test_last_part_of_one_row(gpu, m, n, k, epilogue, dtype):
    near = part_rows(k)
    assert m == near + 1
    rows, epi = [0, 255, near - 257, near - 1, near], dlm.QINT_EPILOGUES[epilogue]
    codes = torch.zeros(m, ref.row_bytes(k), dtype=torch.int8, device=gpu)
    xc, xs = ref.pack(_randn(len(rows), k, seed=1))
    at = torch.tensor(rows, device=gpu)
    codes[at] = xc.to(gpu)
    scales = torch.ones(m, device=gpu)
    scales[at] = xs.to(gpu)
    w, wc, ws = _matrix(gpu, n, k, seed=2)
    cols = n // 2 if epilogue == "swiglu" else n
    y = torch.full((m, cols), 3.0, dtype=dtype, device=gpu)
    assert dlm.qint_linear_workspace(m, w, epi) == 0
    dlm.qint_linear(dlm.make_qint(codes, scales, m, k), w, y, epi, residual=y if epilogue == "add" else None)
    p, bound = ref.product(xc[:, :k], xs, wc, ws)
    if epilogue == "swiglu":
        p, bound = ref.swiglu(p, bound)
    elif epilogue == "add":
        p, bound = 3 + p, bound + ref.U * (3 + p).abs() * (1 + ref.U)
    if dtype == BF16:
        bound = bound + ref.half_ulp(p.abs() + bound, BF16)
    assert bool(((y[at].cpu().double() - p).abs() <= bound).all())
    rest = torch.ones(m, dtype=torch.bool, device=gpu)
    rest[at] = False
    assert bool((y[rest] == (3.0 if epilogue == "add" else 0.0)).all())

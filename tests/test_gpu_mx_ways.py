"""Every way of a product with a 4-bit matrix and every kernel of the attention over a 4-bit
cache, against the 64-bit definition, at sizes for which the planner takes that way (asserted:
a changed constant of the planner fails here instead of leaving a kernel without a test)."""
import pytest
import torch

import mx_reference as ref
from paper_2606_29094_amd import dlm
from test_gpu_mx import Cache, _check_attention

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
FEW, TILE32, TILE64, TILE128, UNPACKED = range(5)


def _matrix(gpu, n, k, seed):
    """A packed matrix of random codes and scales, and its values (64 bits, on the GPU)."""
    gen = torch.Generator(device=gpu).manual_seed(seed)
    g, ld = ref.groups(k), ref.scale_stride(k)
    codes = torch.randint(0, 256, (n, 16 * g), generator=gen, dtype=torch.uint8, device=gpu)
    scales = torch.randint(118, 124, (n, ld), generator=gen, dtype=torch.uint8, device=gpu)
    table = torch.tensor(ref.LEVELS, dtype=torch.float64, device=gpu)
    nib = torch.stack([codes % 16, codes // 16], -1).flatten(1)[:, :k].long()
    w = torch.cat([table, -table])[nib]
    w *= 2.0 ** (scales.double().repeat_interleave(32, 1)[:, :k] - 127)
    return dlm.make_mx(codes, scales, n, k), w


def _check(gpu, m, n, k, dtype, epilogue, plan, pad=0, out_pad=0):
    epi, cols = dlm.MX_EPILOGUES[epilogue], n // 2 if epilogue == "swiglu" else n
    aligned = (1 if (k + pad) % 8 == 0 and k % 8 == 0 else 0) + (2 if (cols + out_pad) % 8 == 0 else 0)
    assert dlm.debug_mx_linear_plan(dtype, m, n, k, epi, k + pad, aligned)[:2] == plan
    q, w = _matrix(gpu, n, k, seed=m)
    gen = torch.Generator(device=gpu).manual_seed(k)
    x = torch.randn(m, k + pad, generator=gen, device=gpu).to(dtype)[:, :k]
    ydt = dtype if epilogue == "swiglu" else F32
    y = torch.randn(m, cols + out_pad, generator=gen, device=gpu).to(ydt)
    before = y.clone()
    need = dlm.mx_linear_workspace(dtype, m, q, epi)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=gpu)
    dlm.mx_linear(x, q, y[:, :cols], epi, ws)
    assert bool((ws[need:] == 0xFF).all()) and torch.equal(y[:, cols:], before[:, cols:])
    xx = x.double()
    want, bound = xx @ w.T, ref.product_bound(xx, w, dtype)
    if epilogue == "swiglu":
        (g, u), (tg, tu) = want.chunk(2, -1), bound.chunk(2, -1)
        want, bound = ref.silu_mul(g, u), ref.swiglu_bound(g, u, tg, tu, dtype)
    elif epilogue == "add":
        want = want + before[:, :cols].double()
        bound = bound + ref.U * want.abs()
    err = (y[:, :cols].double() - want).abs()
    assert bool((err <= bound + 1e-37).all()), float((err / (bound + 1e-37)).max())
    again = before.clone()
    dlm.mx_linear(x, q, again[:, :cols], epi, ws)
    assert torch.equal(again, y)


# rows, n, k, (way, K slices)
BF16_WAYS = [
    (16, 4098, 600, (FEW, 1)), (40, 1030, 8200, (FEW, 6)),
    (263, 66, 264, (TILE32, 1)), (263, 66, 256, (TILE32, 1)), (70, 2050, 4072, (TILE32, 4)),
    (263, 3590, 264, (TILE64, 1)), (35, 24578, 4100, (TILE64, 2)), (35, 8194, 5000, (TILE64, 4)),
    (35, 4098, 9000, (TILE64, 6)),
    (515, 12290, 264, (TILE128, 1)), (515, 12290, 1024, (TILE128, 1)), (70, 24578, 9000, (TILE128, 2)),
    (70, 12290, 9000, (TILE128, 4)), (70, 12290, 8992, (TILE128, 4))]
F32_WAYS = [
    (16, 4098, 600, (FEW, 1)), (263, 66, 264, (TILE32, 1)), (263, 1030, 600, (TILE32, 2)),
    (263, 3590, 264, (TILE64, 1)), (263, 3590, 1288, (TILE64, 2)),
    (515, 1030, 2056, (TILE64, 4)), (263, 1030, 4100, (TILE64, 7)), (263, 1030, 4096, (TILE64, 8)),
    (515, 12290, 264, (TILE128, 1)), (515, 12290, 1024, (TILE128, 1)), (70, 24578, 4100, (TILE128, 2)),
    (70, 12290, 4100, (TILE128, 4)), (70, 12290, 4096, (TILE128, 4))]


@pytest.mark.parametrize("epilogue", ["store", "add", "swiglu"])
@pytest.mark.parametrize("m,n,k,plan", BF16_WAYS)
def test_linear_way(gpu, m, n, k, plan, epilogue):
    _check(gpu, m, n, k, BF16, epilogue, plan)


@pytest.mark.parametrize("epilogue", ["store", "add", "swiglu"])
@pytest.mark.parametrize("m,n,k,plan", F32_WAYS)
def test_linear_way_fp32(gpu, m, n, k, plan, epilogue):
    _check(gpu, m, n, k, F32, epilogue, plan)


@pytest.mark.parametrize("epilogue", ["store", "add"])
@pytest.mark.parametrize("m,n,k,plan", [(515, 12289, 264, (TILE128, 1)), (70, 12291, 9000, (TILE128, 4)),
                                        (263, 3587, 264, (TILE64, 1))])
def test_linear_odd_and_strided(gpu, m, n, k, plan, epilogue):
    _check(gpu, m, n, k, BF16, epilogue, plan, pad=3, out_pad=2)


@pytest.mark.parametrize("epilogue", ["store", "add", "swiglu"])
@pytest.mark.parametrize("m,n,k,pad", [(2050, 4128, 2112, 0), (2300, 8224, 1088, 8)])
def test_linear_unpacked(gpu, m, n, k, pad, epilogue):
    _check(gpu, m, n, k, BF16, epilogue, (UNPACKED, 1), pad=pad)


LARGE = [(397, 397), (390, 400), (400, 385), (397, 397), (397, 321), (3, 0)]


# (rows, keys) of the requests, (kernel, key splits)
@pytest.mark.parametrize("dtype,hq,hkv,dh,reqs,plan", [
    (BF16, 8, 8, 128, [(40, 1200), (39, 1151), (33, 1111), (5, 0)] * 4, (0, 1)),
    (BF16, 5, 5, 64, [(17, 330), (1, 64), (5, 0), (33, 129)], (0, 1)),
    (BF16, 4, 2, 64, [(3, 4000), (2, 70)], (0, 16)),
    (BF16, 7, 1, 128, [(17, 330), (1, 64), (5, 0), (33, 129)], (1, 8)),
    (BF16, 4, 2, 128, [(3, 4000), (2, 70)], (1, 16)),
    (BF16, 16, 16, 64, [(300, 300), (299, 300), (301, 301)], (1, 1)),
    (BF16, 28, 4, 128, [(400, 400), (129, 129), (64, 333), (3, 0)], (1, 1)),
    (BF16, 28, 4, 128, LARGE, (2, 1)), (BF16, 28, 4, 64, LARGE, (2, 1)),
    (BF16, 32, 32, 128, [(400, 400), (399, 391), (390, 400), (400, 385)], (2, 1)),
    (BF16, 28, 4, 128, [(64, 1000), (61, 700)] * 16, (2, 1)),
    (F32, 8, 8, 128, [(40, 1200), (39, 1151), (33, 1111), (5, 0)] * 4, (0, 1)),
    (F32, 4, 2, 64, [(3, 4000), (2, 70)], (0, 16))])
def test_attention_kernel(gpu, dtype, hq, hkv, dh, reqs, plan):
    rows, lens = [m for m, _ in reqs], [l for _, l in reqs]
    assert dlm.debug_mx_attention_plan(dtype, hq, hkv, dh, rows, lens) == plan
    c = Cache(gpu, hq, hkv, dh, dtype, len(reqs), max(lens))
    _check_attention(gpu, c, [(s, l, 0, m) for s, (m, l) in enumerate(reqs)], seed=dh)
    c.close()

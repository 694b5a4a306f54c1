"""Every way of a product with a 4-bit matrix, and the attention kernels, captured into a graph:
each replay, between eager calls on other inputs, gives the eager call's bits."""
import pytest
import torch

from paper_2606_29094_amd import dlm
from test_gpu_mx import Cache, _randn
from test_gpu_mx_ways import BF16, F32, FEW, TILE32, TILE64, TILE128, UNPACKED, _matrix

pytestmark = pytest.mark.gpu


def _replays(inputs, call, result):
    """call() reads what inputs(seed) wrote; result() copies its outputs."""
    want = {}
    for seed in (1, 2, 3):
        inputs(seed)
        call()
        torch.cuda.synchronize()
        want[seed] = result()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for seed in (2, 1, 3, 1):
        inputs(seed)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(result(), want[seed]), seed
        inputs(3)
        call()                              # an eager call between the replays
        assert torch.equal(result(), want[3])


@pytest.mark.parametrize("epilogue", ["store", "add", "swiglu"])
@pytest.mark.parametrize("dtype,m,n,k,way", [
    (BF16, 5, 4098, 600, FEW), (BF16, 40, 1030, 8200, FEW), (BF16, 70, 2050, 4072, TILE32),
    (BF16, 35, 8194, 5000, TILE64), (BF16, 263, 3590, 257, TILE64), (BF16, 515, 12290, 264, TILE128),
    (BF16, 2050, 4128, 2112, UNPACKED), (F32, 5, 4098, 600, FEW), (F32, 515, 1030, 2056, TILE64)])
def test_product(gpu, dtype, m, n, k, way, epilogue):
    epi = dlm.MX_EPILOGUES[epilogue]
    assert dlm.debug_mx_linear_plan(dtype, m, n, k, epi, aligned=3 if k % 8 == 0 else 2)[0] == way
    q, _ = _matrix(gpu, n, k, seed=1)
    cols = n // 2 if epilogue == "swiglu" else n
    x = torch.empty(m, k, dtype=dtype, device=gpu)
    y = torch.empty(m, cols, dtype=dtype if epilogue == "swiglu" else F32, device=gpu)
    ws = torch.empty(max(256, dlm.mx_linear_workspace(dtype, m, q, epi)), dtype=torch.uint8, device=gpu)

    def inputs(seed):
        x.copy_(_randn(m, k, seed=seed))
        y.copy_(_randn(m, cols, seed=seed + 9))
        ws.fill_(seed)

    _replays(inputs, lambda: dlm.mx_linear(x, q, y, epi, ws), y.clone)


@pytest.mark.parametrize("dtype,hq,hkv,dh,reqs", [
    (BF16, 5, 5, 64, [(17, 330), (1, 64), (5, 0)]), (BF16, 7, 1, 128, [(17, 330), (5, 0), (33, 129)]),
    (BF16, 4, 2, 128, [(3, 4000), (2, 70)]), (BF16, 64, 1, 64, [(9, 200), (70, 65)]),
    (BF16, 28, 4, 128, [(397, 397), (390, 400), (400, 385), (397, 397), (397, 321)]),
    (F32, 4, 2, 64, [(3, 4000), (2, 70)])])
def test_attention(gpu, dtype, hq, hkv, dh, reqs):
    c = Cache(gpu, hq, hkv, dh, dtype, len(reqs), max(l for _, l in reqs))
    n = sum(m for m, _ in reqs)
    rows = dlm.make_kv_rows([(s, l, 0, m) for s, (m, l) in enumerate(reqs)])
    q = torch.empty(n, hq * dh, dtype=dtype, device=gpu)
    out = torch.empty_like(q)
    ws = torch.empty(max(256, dlm.mx_kv_attention_workspace(c.handle, rows)), dtype=torch.uint8, device=gpu)
    for s, (_, length) in enumerate(reqs):
        c.fill(s, length, seed=s)
    def inputs(seed):
        q.copy_(_randn(n, hq * dh, seed=seed))
        out.fill_(seed)
        ws.fill_(seed)

    _replays(inputs, lambda: dlm.mx_kv_attention(c.handle, 0, rows, q, out, ws), out.clone)
    c.close()

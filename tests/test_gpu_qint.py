"""Operators on 8-bit integers against their 64-bit definitions (qint_reference)."""
import math

import pytest
import torch

import qint_reference as ref
from paper_2606_29094_amd import dlm

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _randn(*shape, seed=0, dtype=F32, std=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


def _empty(gpu, n, k):
    """Buffers of an [n, k] matrix that hold something else."""
    return dlm.make_qint(torch.full((n, ref.row_bytes(k)), 0x5A, dtype=torch.int8, device=gpu),
                         torch.full((n,), -7.0, device=gpu), n, k)


def _matrix(gpu, n, k, seed=0, std=1.0, x=None):
    """An 8-bit matrix on the GPU with its codes and scales (CPU)."""
    codes, scales = ref.pack(_randn(n, k, seed=seed, std=std) if x is None else x)
    return dlm.make_qint(codes.to(gpu), scales.to(gpu), n, k), codes[:, :k], scales


def _held(q):
    return q._keep[0].cpu(), q._keep[1].cpu()


# ------------------------------------------------------------ pack, unpack
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,k,pad", [(1, 1, 0), (3, 127, 0), (5, 128, 7), (7, 129, 0), (16, 512, 0),
                                     (17, 688, 8), (300, 1031, 1), (6, 4096, 0), (4, 18944, 0),
                                     (2, 16385, 0), (3, 40000, 8), (2, ref.MAX_K, 3)])
def test_pack_unpack(gpu, n, k, pad, dtype):
    big = (_randn(n, k + pad, seed=n + k) * torch.logspace(-44, 37, n)[:, None]).to(dtype)
    x = big[:, :k]
    q = _empty(gpu, n, k)
    dlm.qint_pack(big.to(gpu)[:, :k], q)
    codes, scales = _held(q)
    ref.check_packed(codes, scales, x.double())
    for dt in (F32, BF16):
        out = torch.full((n, k + pad), 7.0, dtype=dt, device=gpu)
        dlm.qint_unpack(q, out[:, :k])
        want = (codes[:, :k].float() * scales[:, None]).to(dt)     # one rounding, then the type's
        assert torch.equal(out[:, :k].cpu(), want)
        assert bool((out[:, k:] == 7.0).all())


def test_pack_borders_and_non_finite(gpu):
    """Ties of rows whose step is a power of two, both ends of the scales, zeros of both signs; a
    row with an infinity or a NaN becomes NaN alone."""
    half = torch.arange(-127, 127).float() + 0.5
    near = torch.cat([half, torch.nextafter(half, torch.tensor(999.0)), torch.nextafter(half, torch.tensor(-999.0))])
    row = torch.cat([near, torch.tensor([127.0, -127.0])])
    rows = [row * 2.0 ** e for e in (-132, -120, -20, 0, 3, 119)]       # (2^-126 is the smallest step)
    ties = len(rows)
    z = torch.zeros_like(row)
    for v in (0.0, -0.0, 1e-45, 2.0 ** -126, 3.4e38):
        rows.append(torch.where(torch.arange(len(row)) == 5, torch.tensor(v), z))
    for v in (math.inf, -math.inf, math.nan):
        r = _randn(len(row), seed=3)
        r[len(row) - 1] = v
        rows.append(r)
    rows.append(_randn(len(row), seed=4))
    x = torch.stack(rows)
    q = _empty(gpu, *x.shape)
    dlm.qint_pack(x.to(gpu), q)
    codes, scales = _held(q)
    ref.check_packed(codes, scales, x.double(), like=torch.arange(ties))
    assert int(scales.isnan().sum()) == 3 and not scales[-1].isnan()
    out = torch.empty(x.shape, device=gpu)
    dlm.qint_unpack(q, out)
    assert bool(out[-4:-1].isnan().all()) and not bool(out[-1].isnan().any())


def test_pack_sees_every_position(gpu):
    """The largest magnitude wherever it stands."""
    for k in (700, 5000, 20000):
        at = torch.arange(0, k, max(1, k // 61))
        x = _randn(len(at), k, seed=k)
        x[torch.arange(len(at)), at] = 1e3
        q = _empty(gpu, len(at), k)
        dlm.qint_pack(x.to(gpu), q)
        ref.check_packed(*_held(q), x.double())


def test_unpack_every_code(gpu):
    codes = torch.arange(-128, 128).to(torch.int8).reshape(1, 256).repeat(4, 1)
    scales = torch.tensor([1.0, 2.0 ** -126, 3.3e-3, 1e36])
    q = dlm.make_qint(codes.to(gpu), scales.to(gpu), 4, 256)
    for dt in (F32, BF16):
        out = torch.empty(4, 256, dtype=dt, device=gpu)
        dlm.qint_unpack(q, out)
        assert torch.equal(out.cpu(), (codes.float() * scales[:, None]).to(dt))


def test_no_rows(gpu):
    q = dlm.make_qint(torch.empty(0, 128, dtype=torch.int8, device=gpu), torch.empty(0, device=gpu), 0, 70)
    w, _, _ = _matrix(gpu, 24, 70)
    dlm.qint_pack(torch.empty(0, 70, device=gpu), q)
    dlm.qint_unpack(q, torch.empty(0, 70, device=gpu))
    dlm.qint_norm(torch.empty(0, 70, device=gpu), torch.ones(70, device=gpu), 1e-5, q)
    assert dlm.qint_linear_workspace(0, w) == 0
    dlm.qint_linear(q, w, torch.empty(0, 24, device=gpu))


# -------------------------------------------------------------------- norm
def _check_norm(gpu, n, k, splits, dtype, out, pad=0, seed=0, std=1.0, eps=1e-5, like=None):
    h = _randn(n, k + pad, seed=seed, std=std)
    g = 1 + _randn(k, seed=seed + 1, std=0.2)
    add = _randn(splits, n, k + pad, seed=seed + 2, dtype=dtype) if splits else None
    want = h[:, :k].clone()
    for s in range(splits):
        want = want + add[s, :, :k].float()                  # fp32, in order
    hd, q = h.to(gpu), _empty(gpu, n, k)
    od = torch.full((n, k + pad), 9.0, device=gpu) if out == "other" else hd
    ad = None if add is None else add.to(gpu)[:, :, :k]
    if splits == 1 and pad == 0:
        ad = ad[0]
    call = lambda: dlm.qint_norm(hd[:, :k], g.to(gpu), eps, q, add=ad,
                                 h_out=od[:, :k] if out == "other" else None)
    call()
    assert torch.equal(od[:, :k].cpu(), want)
    if out == "other":
        assert torch.equal(hd.cpu(), h)
    if pad:
        assert torch.equal(od[:, k:].cpu(), (torch.full((n, pad), 9.0) if out == "other" else h[:, k:]))
    x = want.double()
    y = x / torch.sqrt((x * x).mean(1, keepdim=True) + torch.tensor(eps).double()) * g.double()
    codes, scales = _held(q)
    ref.check_packed(codes, scales, y)
    if out == "other":
        call()
        assert torch.equal(_held(q)[0], codes) and torch.equal(_held(q)[1], scales)


@pytest.mark.parametrize("out", ["in place", "other"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("splits", [0, 1, 2, 3, 8])
@pytest.mark.parametrize("n,k", [(1, 4096), (5, 3584), (600, 256), (2, 16640)])
def test_norm(gpu, n, k, splits, dtype, out):
    _check_norm(gpu, n, k, splits, dtype, out, seed=n + k + splits)


@pytest.mark.parametrize("splits", [0, 1, 4])
@pytest.mark.parametrize("n,k,pad", [(1, 1, 0), (3, 2, 1), (4, 63, 0), (5, 255, 2), (7, 1031, 0), (700, 130, 0),
                                     (600, 4092, 4), (3, 4100, 3), (2, 16385, 0), (2, 20001, 0), (1, ref.MAX_K, 1)])
def test_norm_shapes(gpu, n, k, pad, splits):
    for dtype in (BF16, F32):
        for out in ("in place", "other"):
            _check_norm(gpu, n, k, splits, dtype, out, pad=pad, seed=k)


@pytest.mark.parametrize("std,eps", [(1e-20, 1e-5), (1e-20, 1e-38), (1e30, 1e-5), (1.0, 1e30), (3.0, 1e-45)])
def test_norm_magnitudes(gpu, std, eps):
    """Squares that leave fp32's range, an eps that outweighs them."""
    _check_norm(gpu, 9, 700, 0, F32, "in place", std=std, eps=eps)
    _check_norm(gpu, 3, 17000, 1, F32, "other", std=std, eps=eps)


def test_norm_rows_of_zeros_and_non_finite(gpu):
    n, k = 8, 600
    h, g = _randn(n, k, seed=1), 1 + _randn(k, seed=2, std=0.1)
    h[1] = 0
    h[2, 599], h[3, 0], h[4, 300] = math.inf, -math.inf, math.nan
    g[77] = 0                                   # a channel that is switched off
    q = _empty(gpu, n, k)
    dlm.qint_norm(h.to(gpu), g.to(gpu), 1e-5, q)
    codes, scales = _held(q)
    x = h.double()
    y = x / torch.sqrt((x * x).mean(1, keepdim=True) + torch.tensor(1e-5).double()) * g.double()
    y[2:5] = math.nan
    ref.check_packed(codes, scales, y)
    assert not codes[1].any() and scales[1] == 2.0 ** -126
    g[5] = math.nan                              # a gain: every row
    dlm.qint_norm(h.to(gpu), g.to(gpu), 1e-5, q)
    assert bool(_held(q)[1].isnan().all()) and not _held(q)[0].any()


def test_norm_without_a_place_for_the_sum(gpu):
    """h_out NULL: the sum is normed and nothing but the packed rows is written."""
    import ctypes
    for n, k in ((5, 640), (3, 16500)):
        h, a, g = _randn(n, k, seed=1), _randn(2, n, k, seed=2), 1 + _randn(k, seed=3, std=0.1)
        hd, ad, gd, q = h.to(gpu), a.to(gpu), g.to(gpu), _empty(gpu, n, k)
        st = torch.cuda.current_stream().cuda_stream
        dlm.check(dlm.lib().dlm_qint_norm(hd.data_ptr(), k, None, 0, dlm.DLM_F32, ad.data_ptr(), 2, n * k, k,
                                          gd.data_ptr(), 1e-5, ctypes.byref(q), st))
        assert torch.equal(hd.cpu(), h) and torch.equal(ad.cpu(), a)
        x = (h + a[0] + a[1]).double()
        ref.check_packed(*_held(q), x / torch.sqrt((x * x).mean(1, keepdim=True) + torch.tensor(1e-5).double()) *
                         g.double())


# ---------------------------------------------------------------- products
def _check_linear(gpu, m, n, k, epilogue, dtype=F32, pad=0, seed=0, x=None, w=None, in_place=False, guard=4096):
    xq, xc, xs = x if x else _matrix(gpu, m, k, seed=seed + 1, std=2.0)
    wq, wc, ws = w if w else _matrix(gpu, n, k, seed=seed)
    epi = dlm.QINT_EPILOGUES[epilogue]
    cols = n // 2 if epilogue == "swiglu" else n
    y = _randn(m, cols + pad, seed=seed + 2).to(dtype).to(gpu)
    before = y.cpu()
    r = None
    if epilogue == "add":
        r = y[:, :cols] if in_place else _randn(m, cols + 3, seed=seed + 3).to(gpu)[:, :cols]
    res = None if r is None else r.cpu().double()
    need = dlm.qint_linear_workspace(m, wq, epi)
    ws_t = torch.full((need + guard,), 0xFF, dtype=torch.uint8, device=gpu)
    dlm.qint_linear(xq, wq, y[:, :cols], epi, ws_t, residual=r)
    got = y.cpu()
    assert torch.equal(got[:, cols:], before[:, cols:])
    assert bool((ws_t[need:] == 0xFF).all())
    p, bound = ref.product(xc, xs, wc, ws)
    if epilogue == "swiglu":
        p, bound = ref.swiglu(p, bound)
    elif epilogue == "add":
        p = res + p
        bound = bound + ref.U * p.abs() * (1 + ref.U) + 2.0 ** -149
    if dtype == BF16:
        bound = bound + ref.half_ulp(p.abs() + bound, BF16)
    err = (got[:, :cols].double() - p).abs()
    assert bool((err <= bound + 2.0 ** -140).all()), float((err / (bound + 2.0 ** -140)).max())
    return got[:, :cols]


@pytest.mark.parametrize("epilogue,dtype", [("store", F32), ("store", BF16), ("add", F32), ("swiglu", F32),
                                            ("swiglu", BF16)])
@pytest.mark.parametrize("m", [1, 5, 16, 17, 32, 33, 64, 65, 130, 257])
def test_linear_rows(gpu, m, epilogue, dtype):
    _check_linear(gpu, m, 160, 512, epilogue, dtype, seed=m)


@pytest.mark.parametrize("epilogue,dtype", [("store", F32), ("add", F32), ("swiglu", BF16)])
@pytest.mark.parametrize("n,k", [(2, 1), (18, 31), (34, 64), (66, 127), (130, 129), (256, 688), (94, 1031),
                                 (688, 264), (4096, 256), (512, 4096), (1376, 256)])
def test_linear_shapes(gpu, n, k, epilogue, dtype):
    for m in (3, 70):
        _check_linear(gpu, m, n, k, epilogue, dtype, seed=n)


@pytest.mark.parametrize("m", [3, 70, 300])
@pytest.mark.parametrize("pad", [1, 2, 5, 8])
def test_linear_strides(gpu, m, pad):
    for epilogue, dtype in (("store", F32), ("store", BF16), ("add", F32), ("swiglu", F32), ("swiglu", BF16)):
        _check_linear(gpu, m, 258, 320, epilogue, dtype, pad=pad, seed=pad)
    _check_linear(gpu, m, 258, 320, "add", F32, pad=pad, seed=pad, in_place=True)


@pytest.mark.parametrize("m", [1, 40, 260])
def test_linear_odd_columns(gpu, m):
    for n in (1, 17, 33, 257):
        _check_linear(gpu, m, n, 200, "store", BF16, seed=n)
        _check_linear(gpu, m, n, 200, "add", F32, seed=n)
        _check_linear(gpu, m, 2 * n, 200, "swiglu", BF16, seed=n)


def test_linear_largest_sums(gpu):
    """Every code -128, the longest rows: 2^14 * 131071 in a 32-bit sum."""
    k = ref.MAX_K
    codes = torch.zeros(20, ref.row_bytes(k), dtype=torch.int8)
    codes[:, :k] = -128
    one = torch.ones(20)
    mk = lambda: (dlm.make_qint(codes.to(gpu), one.to(gpu), 20, k), codes[:, :k], one)
    y = _check_linear(gpu, 20, 20, k, "store", F32, x=mk(), w=mk())
    assert float(y[0, 0]) == 2.0 ** 14 * k // 128 * 128      # (rounded to fp32's step of 128)


def test_linear_scales_of_any_size(gpu):
    """Scales from the smallest to the largest, tokens against channels; a product inside the
    range of fp32 is neither lost nor made infinite on the way to it."""
    m, n, k = 40, 48, 160
    sx, sw = torch.logspace(-37.9, 36, m), torch.logspace(-37.9, 36, n)
    xc, wc = ref.pack(_randn(m, k, seed=1))[0], ref.pack(_randn(n, k, seed=2))[0]
    xq, wq = dlm.make_qint(xc.to(gpu), sx.to(gpu), m, k), dlm.make_qint(wc.to(gpu), sw.to(gpu), n, k)
    y = torch.empty(m, n, device=gpu)
    dlm.qint_linear(xq, wq, y)
    p, bound = ref.product(xc[:, :k], sx, wc[:, :k], sw)
    inside = p.abs() < 3.4e38
    got = y.cpu().double()
    assert bool(((got - p).abs() <= bound + 2.0 ** -149)[inside].all())
    assert bool((got.abs() == math.inf)[p.abs() > 3.41e38].all()) and bool((~inside).any())


def test_linear_nan_rows_stay_alone(gpu):
    m, n, k = 37, 50, 300
    x = _randn(m, k, seed=1)
    x[4, 7] = math.nan
    w = _randn(n, k, seed=2)
    w[11, 0] = math.inf
    xq, wq = _empty(gpu, m, k), _empty(gpu, n, k)
    dlm.qint_pack(x.to(gpu), xq)
    dlm.qint_pack(w.to(gpu), wq)
    y = torch.empty(m, n, device=gpu)
    dlm.qint_linear(xq, wq, y)
    nan = torch.zeros(m, n, dtype=torch.bool)
    nan[4], nan[:, 11] = True, True
    assert torch.equal(y.cpu().isnan(), nan)


@pytest.mark.parametrize("n,k,epilogue", [(700, 1100, "store"), (4096, 4096, "swiglu"), (258, 12288, "add")])
def test_linear_rows_alone_and_together(gpu, n, k, epilogue):
    """A row gives the same bits in every batch."""
    big = 700
    xq, xc, xs = _matrix(gpu, big, k, seed=5)
    wq, wc, ws = _matrix(gpu, n, k, seed=6)
    epi = dlm.QINT_EPILOGUES[epilogue]
    cols = n // 2 if epilogue == "swiglu" else n
    r = _randn(big, cols, seed=7).to(gpu)

    def some(lo, hi):
        part = dlm.make_qint(xq._keep[0][lo:hi], xq._keep[1][lo:hi], hi - lo, k)
        y = torch.empty(hi - lo, cols, device=gpu)
        ws_t = torch.empty(max(1, dlm.qint_linear_workspace(hi - lo, wq, epi)), dtype=torch.uint8, device=gpu)
        dlm.qint_linear(part, wq, y, epi, ws_t, residual=r[lo:hi])
        return y

    whole = some(0, big)
    for lo, hi in ((0, 1), (699, 700), (3, 19), (100, 133), (200, 290), (5, 260), (0, 513)):
        assert torch.equal(some(lo, hi), whole[lo:hi]), (lo, hi)


# ------------------------------------------------------------ together
def test_a_layer_of_them(gpu):
    """Norm, gate/up, packing, down into the residual: each step on what the step before gave."""
    m, d, f = 45, 320, 500
    h, add, g = _randn(m, d, seed=1), _randn(m, d, seed=2, dtype=BF16), 1 + _randn(d, seed=3, std=0.1)
    wg, wgc, wgs = _matrix(gpu, 2 * f, d, seed=4, std=0.05)
    wd, wdc, wds = _matrix(gpu, d, f, seed=5, std=0.05)
    hd, x, a = h.to(gpu), _empty(gpu, m, d), _empty(gpu, m, f)
    act = torch.empty(m, f, dtype=BF16, device=gpu)
    ws = torch.empty(max(dlm.qint_linear_workspace(m, wg, dlm.DLM_QINT_SWIGLU),
                         dlm.qint_linear_workspace(m, wd, dlm.DLM_QINT_ADD), 1), dtype=torch.uint8, device=gpu)

    def layer():
        dlm.qint_norm(hd, g.to(gpu), 1e-5, x, add=add.to(gpu))
        dlm.qint_linear(x, wg, act, dlm.DLM_QINT_SWIGLU, ws)
        dlm.qint_pack(act, a)
        dlm.qint_linear(a, wd, hd, dlm.DLM_QINT_ADD, ws, residual=hd)

    layer()
    h1 = h + add.float()
    y = h1.double() / torch.sqrt((h1.double() ** 2).mean(1, keepdim=True) + torch.tensor(1e-5).double()) * g.double()
    xc, xs = _held(x)
    ref.check_packed(xc, xs, y)
    want, bound = ref.swiglu(*ref.product(xc[:, :d], xs, wgc, wgs))
    err = (act.cpu().double() - want).abs()
    assert bool((err <= bound + ref.half_ulp(want.abs() + bound, BF16)).all())
    ac, as_ = _held(a)
    ref.check_packed(ac, as_, act.cpu().double())
    p, bound = ref.product(ac[:, :f], as_, wdc, wds)
    want = h1.double() + p
    assert bool(((hd.cpu().double() - want).abs() <= bound + ref.U * want.abs() * 1.001).all())

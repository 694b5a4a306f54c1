"""8-bit integers on the host: the format's reference, buffer sizes, and every call that is
refused before anything is enqueued (the addresses below are never used)."""
import ctypes
import math
import os

import pytest
import torch

import qint_reference as ref
from paper_2606_29094_amd import dlm

FAKE = 0x100000
E, BIG = dlm.DLM_EINVAL, dlm.DLM_EUNSUPPORTED
pytestmark = pytest.mark.skipif(not os.path.exists(dlm.LIB_PATH), reason="libdlm.so not built")


def test_reference_values():
    x = torch.tensor([[127, 0.5, 1.5, -2.5, 126.51, 0, 0], [0, 0, 0, 0, 0, 0, -0.0], [1e-45] + [0] * 6,
                      [254, 1, 3, -5, 2, 0, 0], [math.nan, 1, 2, 3, 4, 5, 6]])
    codes, scales = ref.pack(x)
    assert codes.shape == (5, 128) and not codes[:, 7:].any()
    assert codes[0, :7].tolist() == [127, 0, 2, -2, 127, 0, 0] and scales[0] == 1
    assert codes[3, :5].tolist() == [127, 0, 2, -2, 1] and scales[3] == 2
    assert scales[1] == scales[2] == 2.0 ** -126 and not codes[1:3].any()
    assert scales[4].isnan() and not codes[4].any()
    ref.check_packed(codes, scales, x.double())
    for wrong in (codes + torch.eye(5, 128, dtype=torch.int8), torch.roll(codes, 1, 1)):
        with pytest.raises(AssertionError):
            ref.check_packed(wrong, scales, x.double())
    with pytest.raises(AssertionError):
        ref.check_packed(codes, scales * (1 + 2.0 ** -22), x.double())


@pytest.mark.parametrize("n,k,codes", [(0, 5, 0), (1, 1, 128), (3, 128, 384), (3, 129, 768),
                                       (7, ref.MAX_K, 7 * 131072)])
def test_buffer_sizes(n, k, codes):
    assert dlm.qint_bytes(n, k) == (codes, 4 * n)


def _q(n=64, k=64, codes=FAKE, scales=FAKE):
    return dlm.DlmQint(codes, scales, n, k)


def _norm(L, h=FAKE, ldh=64, out=FAKE, ldo=64, dtype=1, add=FAKE, splits=2, stride=64 * 64, ldadd=64, gain=FAKE,
          eps=1e-5, q=None):
    return L.dlm_qint_norm(h, ldh, out, ldo, dtype, add, splits, stride, ldadd, gain, eps, q or _q(), None)


def _linear(L, x=None, w=None, epilogue=0, res=FAKE, ldr=64, dtype=0, y=FAKE, ldy=64, ws=FAKE, size=1 << 40):
    return L.dlm_qint_linear(x or _q(4), w or _q(), epilogue, res, ldr, dtype, y, ldy, ws, size, None)


@pytest.mark.parametrize("call,status", [
    (lambda L: L.dlm_qint_bytes(-1, 4, None, None), E),
    (lambda L: L.dlm_qint_bytes(4, 0, None, None), E),
    (lambda L: L.dlm_qint_bytes(4, ref.MAX_K + 1, None, None), BIG),
    (lambda L: L.dlm_qint_pack(5, FAKE, 64, _q(), None), E),
    (lambda L: L.dlm_qint_pack(1, None, 64, _q(), None), E),
    (lambda L: L.dlm_qint_pack(1, FAKE, 63, _q(), None), E),
    (lambda L: L.dlm_qint_pack(1, FAKE, 64, None, None), E),
    (lambda L: L.dlm_qint_pack(1, FAKE, 64, _q(codes=None), None), E),
    (lambda L: L.dlm_qint_pack(1, FAKE, 64, _q(scales=None), None), E),
    (lambda L: L.dlm_qint_pack(1, FAKE, 64, _q(codes=FAKE + 8), None), E),
    (lambda L: L.dlm_qint_pack(1, FAKE, 64, _q(scales=FAKE + 2), None), E),
    (lambda L: L.dlm_qint_pack(1, FAKE, 64, _q(n=-1), None), E),
    (lambda L: L.dlm_qint_pack(1, FAKE, 64, _q(k=0), None), E),
    (lambda L: L.dlm_qint_pack(1, FAKE, 1 << 40, _q(k=ref.MAX_K + 1), None), BIG),
    (lambda L: L.dlm_qint_unpack(_q(), 2, FAKE, 64, None), E),
    (lambda L: L.dlm_qint_unpack(_q(), 1, None, 64, None), E),
    (lambda L: L.dlm_qint_unpack(_q(), 1, FAKE, 10, None), E),
    (lambda L: L.dlm_qint_unpack(None, 1, FAKE, 64, None), E),
    (lambda L: _norm(L, h=None), E), (lambda L: _norm(L, gain=None), E), (lambda L: _norm(L, add=None), E),
    (lambda L: _norm(L, ldh=63), E), (lambda L: _norm(L, ldo=63), E), (lambda L: _norm(L, ldadd=63), E),
    (lambda L: _norm(L, stride=-1), E), (lambda L: _norm(L, splits=-1), E), (lambda L: _norm(L, dtype=2), E),
    (lambda L: _norm(L, ldo=128), E),            # in place, another stride
    (lambda L: _norm(L, eps=0.0), E), (lambda L: _norm(L, eps=-1.0), E), (lambda L: _norm(L, eps=math.inf), E),
    (lambda L: _norm(L, eps=math.nan), E), (lambda L: _norm(L, q=_q(codes=FAKE + 4)), E),
    (lambda L: _norm(L, ldh=1 << 20, ldo=1 << 20, ldadd=1 << 20, q=_q(k=1 << 18)), BIG),
    (lambda L: L.dlm_qint_linear_workspace(4, _q(), 0, None), E),
    (lambda L: L.dlm_qint_linear_workspace(-1, _q(), 0, None), E),
    (lambda L: L.dlm_qint_linear_workspace(4, _q(n=0), 0, None), E),
    (lambda L: _linear(L, x=_q(1 << 30)), E), (lambda L: _linear(L, x=_q(4, 65)), E),
    (lambda L: _linear(L, w=_q(0)), E), (lambda L: _linear(L, w=_q(63), epilogue=2), E),
    (lambda L: _linear(L, epilogue=3), E), (lambda L: _linear(L, epilogue=-1), E),
    (lambda L: _linear(L, epilogue=1, dtype=1), E), (lambda L: _linear(L, epilogue=1, res=None), E),
    (lambda L: _linear(L, epilogue=1, ldr=63), E), (lambda L: _linear(L, epilogue=1, ldr=128), E),
    (lambda L: _linear(L, dtype=7), E), (lambda L: _linear(L, y=None), E), (lambda L: _linear(L, ldy=63), E),
    (lambda L: _linear(L, x=_q(4, codes=FAKE + 1)), E), (lambda L: _linear(L, w=_q(codes=None)), E),
    (lambda L: _linear(L, x=_q(4, 131000), w=_q(70000, 131000), ldy=70000), BIG),
    (lambda L: _linear(L, x=_q(4, 131000), w=_q(65505, 131000), ldy=70000), BIG),      # 65536 in whole 32s
    (lambda L: L.dlm_qint_linear_workspace(4, _q(65505, 131000), 0, None), BIG),
    (lambda L: L.dlm_qint_linear_workspace(4, _q(65504, 131000), 0, None), E),         # (no place for the size)
    (lambda L: _linear(L, x=_q(4, 1 << 20), w=_q(64, 1 << 20)), BIG),
])
def test_calls_refused(call, status):
    L = dlm.lib()
    by_ref = lambda x: ctypes.byref(x) if isinstance(x, dlm.DlmQint) else x

    class Through:
        def __getattr__(self, name):
            return lambda *a: getattr(L, name)(*[by_ref(x) for x in a])

    assert call(Through()) == status
    assert dlm.last_error()


def test_no_rows_is_no_work():
    L, none = dlm.lib(), ctypes.byref(_q(0, 64, None, None))
    assert L.dlm_qint_pack(1, None, 64, none, None) == dlm.DLM_OK
    assert L.dlm_qint_unpack(none, 1, None, 64, None) == dlm.DLM_OK
    assert L.dlm_qint_norm(None, 64, None, 64, 0, None, 0, 0, 0, None, 1e-5, none, None) == dlm.DLM_OK
    assert L.dlm_qint_linear(none, ctypes.byref(_q()), 0, None, 0, 0, None, 64, None, 0, None) == dlm.DLM_OK


def test_binding_refuses_host_tensors_and_shapes():
    q, w = _q(8, 64), _q(6, 64)
    f = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)
    for a in [(f(8, 64), q), (f(8, 63), q), (f(8, 64, dtype=torch.float16), q), (f(64, 8).T, q)]:
        with pytest.raises(ValueError):                 # (the first: not in device memory)
            dlm.qint_pack(*a)
        with pytest.raises(ValueError):
            dlm.qint_unpack(a[1], a[0])
    for h, g, add, out in [(f(8, 64), f(64), None, None), (f(8, 64), f(63), None, None),
                           (f(8, 64, dtype=torch.bfloat16), f(64), None, None), (f(8, 64), f(64), f(7, 64), None),
                           (f(8, 64), f(64), f(2, 8, 65), None), (f(8, 64), f(64), None, f(8, 65)),
                           (f(8, 64), f(64), f(8, 64, dtype=torch.int32), None)]:
        with pytest.raises(ValueError):
            dlm.qint_norm(h, g, 1e-5, q, add=add, h_out=out)
    for y, epilogue, res in [(f(8, 6), 0, None), (f(8, 5), 0, None), (f(8, 6), 2, None), (f(8, 6), 1, None),
                             (f(8, 6), 1, f(8, 5)), (f(8, 6), 1, f(8, 6, dtype=torch.bfloat16)),
                             (f(8, 6, dtype=torch.float16), 0, None)]:
        with pytest.raises(ValueError):
            dlm.qint_linear(q, w, y, epilogue, residual=res)
    with pytest.raises(ValueError):
        dlm.make_qint(torch.zeros(8, 128, dtype=torch.int8), f(8), 8, 64)


# ------------------------------------------------------------------ workspace
def test_workspace_is_checked():
    """A product whose K is split: no workspace, an unaligned one, a small one."""
    L, x, w = dlm.lib(), _q(40, 18944), _q(3584, 18944)
    assert dlm.debug_qint_linear_plan(40, 3584, 18944)[1] > 1
    need = dlm.qint_linear_workspace(40, w)
    assert need == 40 * 3584 * 4 * dlm.debug_qint_linear_plan(40, 3584, 18944)[1]
    b = ctypes.byref
    call = lambda ws, size: L.dlm_qint_linear(b(x), b(w), 0, None, 0, 0, FAKE, 3584, ws, size, None)
    assert call(None, need) == E and call(FAKE + 128, need) == E
    assert call(FAKE, need - 1) == dlm.DLM_ESIZE
    assert dlm.qint_linear_workspace(0, w) == 0


def test_plans_are_sound():
    """Plans over a wide range: slices that are not empty and that the scratch holds, tiles that
    the epilogue can run; the hook refuses what the call does."""
    import random
    rng = random.Random(3)
    size = lambda lo, hi: int(lo * (hi / lo) ** rng.random())
    for _ in range(5000):
        m, n, k, e = size(1, 600000) % 524288 + 1, 2 * size(1, 60000), size(1, ref.MAX_K), rng.randrange(3)
        if n * ref.row_bytes(k) > 1 << 33:
            continue
        cfg, slices, sub, group = dlm.debug_qint_linear_plan(m, n, k, e, rng.choice([8, 80, 256, 304]))
        tiles = ref.row_bytes(k) // 128
        assert 1 <= slices <= max(1, tiles)
        if cfg >= 0:
            per = -(-tiles // slices)
            assert -(-tiles // per) == slices                 # none of them empty
            bm, bn, flags = dlm.debug_gemm_info(cfg)
            assert sub == 0 or (flags & sub and slices * sub > 0)
            assert slices > 1 or e != dlm.DLM_QINT_SWIGLU or not flags & 8
            # the tiles' 32-bit offsets: rows beyond them are taken in turn, unsplit
            assert slices == 1 or m * ref.row_bytes(k) // 2 < 1 << 32
        else:
            assert m <= 16
    for bad in [(0, 8, 8, 0), (1, 0, 8, 0), (1, 8, 0, 0), (1, 7, 8, 2), (1, 8, 8, 3), (1 << 20, 8, 8, 0)]:
        with pytest.raises(dlm.DlmError):
            dlm.debug_qint_linear_plan(*bad)
    with pytest.raises(dlm.DlmError):
        dlm.debug_qint_linear_plan(1, 8, 8, 0, 0)
    assert dlm.lib().dlm_debug_qint_linear_plan(1, 8, 8, 0, 256, None) == E


# ----------------------------------------------------------------------- models
def _cfg(**kw):
    c = dict(n_layers=2, d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, d_ffn=688, vocab=2048,
             mask_id=2047, rms_eps=1e-5, rope_theta=1e4, inv_tau=10.0, dtype=dlm.DLM_BF16)
    c.update(kw)
    return dlm.DlmConfig(**c)


def _weights(**kw):
    shapes = dict(w_qkv=(512, 256), w_o=(256, 256), w_gate_up=(1376, 256), w_down=(256, 688))
    shapes.update(kw)
    mk = lambda name: _q(*shapes[name])
    arr = (dlm.DlmLayerQint * 2)(*[dlm.DlmLayerQint(FAKE, mk("w_qkv"), mk("w_o"), FAKE, mk("w_gate_up"),
                                                    mk("w_down")) for _ in range(2)])
    w = dlm.DlmWeightsQint(FAKE, FAKE, FAKE, arr)
    w._keep = arr
    return w


def test_load_model():
    m = dlm.load_weights_qint(_cfg(), _weights())
    assert dlm.workspace_bytes(m, 64, 2) > 0
    assert dlm.kv_cache_alloc_mx(m, 2, 64)[1] > 0 and dlm.kv_cache_alloc(m, 2, 64)[1] > 0
    dlm.model_destroy(m)


@pytest.mark.parametrize("name,shape", [("w_qkv", (511, 256)), ("w_o", (256, 255)), ("w_gate_up", (688, 256)),
                                        ("w_down", (256, 704)), ("w_o", (0, 256))])
def test_load_refuses_other_shapes(name, shape):
    with pytest.raises(dlm.DlmError) as e:
        dlm.load_weights_qint(_cfg(), _weights(**{name: shape}))
    assert e.value.status == E and name in str(e.value)


def test_load_refuses_what_is_missing_or_unsupported():
    for field in ("codes", "scales"):
        w = _weights()
        setattr(w.layers[1].w_o, field, None)
        with pytest.raises(dlm.DlmError) as e:
            dlm.load_weights_qint(_cfg(), w)
        assert "layer 1: w_o" in str(e.value)
    w = _weights()
    w.layers[0].ffn_norm = None
    with pytest.raises(dlm.DlmError):
        dlm.load_weights_qint(_cfg(), w)
    with pytest.raises(dlm.DlmError):
        dlm.load_weights_qint(_cfg(rms_eps=0.0), _weights())
    big = dict(w_gate_up=(2 * 131072, 256), w_down=(256, 131072))
    with pytest.raises(dlm.DlmError) as e:
        dlm.load_weights_qint(_cfg(d_ffn=131072), _weights(**big))
    assert e.value.status == BIG and "w_down" in str(e.value)
    assert dlm.lib().dlm_load_weights_qint(None, None, None) == E


def test_engine_refuses_both_kinds():
    from paper_2606_29094_amd import engine
    with pytest.raises(ValueError):
        engine.DeviceModel(engine.ModelShape(1, 64, 1, 1, 64, 64, 64, "bf16"), {}, 1.0, packed=True, int8=True)

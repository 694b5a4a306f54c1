"""4-bit operands on the host: the format's reference, buffer sizes, and every call
that is refused before anything is enqueued (the addresses below are never used)."""
import ctypes
import os

import pytest
import torch

import mx_reference as ref
from paper_2606_29094_amd import dlm

FAKE = 0x100000
pytestmark = pytest.mark.skipif(not os.path.exists(dlm.LIB_PATH), reason="libdlm.so not built")


def test_reference_values():
    # one group: largest magnitude 7 -> scale 1; borders go to the even code
    x = [7, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -0.75, -6, 0, -0.0]
    w = torch.tensor([x + [0.0] * (40 - len(x))])
    w[0, 32:] = torch.tensor([1e-3, 0, 0, 0, 0, 0, 0, 0])
    codes, scales = ref.pack(w)
    assert codes.shape == (1, 32) and scales.shape == (1, 16)
    assert scales[0, 0] == 127 and scales[0, 2:].sum() == 0
    v = ref.values(codes, scales, 40)[0]
    want = [6, 0, 0.5, 1, 1, 2, 2, 4, 4, 6, -1, -6, 0, 0]
    assert v[:14].tolist() == want
    assert abs(v[32] - 1e-3) < 1e-3 / 7
    assert torch.equal(ref.values(*ref.pack(torch.full((1, 5), float("nan"))), 5).isnan(),
                       torch.ones(1, 5, dtype=torch.bool))


@pytest.mark.parametrize("n,k,codes,scales", [(1, 1, 16, 16), (3, 32, 48, 48), (3, 33, 96, 48),
                                              (7, 512, 7 * 256, 7 * 16), (7, 513, 7 * 272, 7 * 32)])
def test_buffer_sizes(n, k, codes, scales):
    assert dlm.mx_bytes(n, k) == (codes, scales)


def _status(fn, *a):
    return fn(*a)


def _mx(n=64, k=64, codes=FAKE, scales=FAKE):
    return dlm.DlmMx(codes, scales, n, k)


@pytest.mark.parametrize("call,status", [
    (lambda L: L.dlm_mx_bytes(0, 4, None, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_pack(5, FAKE, 64, _mx(), None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_pack(1, None, 64, _mx(), None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_pack(1, FAKE, 63, _mx(), None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_pack(1, FAKE, 64, None, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_pack(1, FAKE, 64, _mx(codes=None), None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_pack(1, FAKE, 64, _mx(codes=FAKE + 8), None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_pack(1, FAKE, 64, _mx(scales=FAKE + 1), None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_pack(1, FAKE, 64, _mx(n=0), None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_pack(1, FAKE, 1 << 40, _mx(k=(1 << 31) - 1), None), dlm.DLM_EUNSUPPORTED),
    (lambda L: L.dlm_mx_unpack(_mx(), 2, FAKE, 64, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_unpack(_mx(), 1, None, 64, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_unpack(_mx(), 1, FAKE, 10, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_linear_workspace(1, 4, _mx(), 0, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_linear(1, FAKE, 64, -1, _mx(), 0, FAKE, 64, None, 0, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_linear(1, FAKE, 64, 1 << 30, _mx(), 0, FAKE, 64, None, 0, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_linear(1, FAKE, 64, 4, _mx(), 3, FAKE, 64, None, 0, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_linear(1, FAKE, 64, 4, _mx(n=63), 2, FAKE, 64, None, 0, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_linear(1, FAKE, 63, 4, _mx(), 0, FAKE, 64, None, 0, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_linear(1, FAKE, 64, 4, _mx(), 0, FAKE, 63, None, 0, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_linear(1, None, 64, 4, _mx(), 0, FAKE, 64, None, 0, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_linear(1, FAKE, 64, 4, _mx(), 0, None, 64, None, 0, None), dlm.DLM_EINVAL),
    # fp32 rows are staged: no workspace, an unaligned one, a small one
    (lambda L: L.dlm_mx_linear(0, FAKE, 64, 4, _mx(), 0, FAKE, 64, None, 1 << 20, None), dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_linear(0, FAKE, 64, 4, _mx(), 0, FAKE, 64, FAKE + 16, 1 << 20, None),
     dlm.DLM_EINVAL),
    (lambda L: L.dlm_mx_linear(0, FAKE, 64, 4, _mx(), 0, FAKE, 64, FAKE, 16, None), dlm.DLM_ESIZE),
])
def test_matrix_calls_refused(call, status):
    L = dlm.lib()
    by_ref = lambda x: ctypes.byref(x) if isinstance(x, dlm.DlmMx) else x

    class Through:
        def __getattr__(self, name):
            return lambda *a: getattr(L, name)(*[by_ref(x) for x in a])

    assert call(Through()) == status
    assert dlm.last_error()


def test_no_rows_is_no_work():
    assert dlm.lib().dlm_mx_linear(1, None, 64, 0, ctypes.byref(_mx()), 0, None, 64, None, 0,
                                   None) == dlm.DLM_OK


def _cfg(**kw):
    c = dict(n_layers=2, d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, d_ffn=688,
             vocab=2048, mask_id=2047, rms_eps=1e-5, rope_theta=1e4, inv_tau=10.0,
             dtype=dlm.DLM_BF16)
    c.update(kw)
    return dlm.DlmConfig(**c)


def _weights(**kw):
    shapes = dict(w_qkv=(512, 256), w_o=(256, 256), w_gate_up=(1376, 256), w_down=(256, 688))
    shapes.update(kw)
    mk = lambda name: _mx(*shapes[name])
    arr = (dlm.DlmLayerMx * 2)(*[dlm.DlmLayerMx(FAKE, mk("w_qkv"), mk("w_o"), FAKE, mk("w_gate_up"),
                                                mk("w_down")) for _ in range(2)])
    w = dlm.DlmWeightsMx(FAKE, FAKE, FAKE, arr)
    w._keep = arr
    return w


def test_load_packed_model():
    m = dlm.load_weights_mx(_cfg(), _weights())
    # the packed model's steps need workspace like any model's
    assert dlm.workspace_bytes(m, 64, 2) > 0
    dlm.model_destroy(m)


@pytest.mark.parametrize("name,shape", [("w_qkv", (511, 256)), ("w_o", (256, 255)),
                                        ("w_gate_up", (688, 256)), ("w_down", (256, 704))])
def test_load_refuses_other_shapes(name, shape):
    with pytest.raises(dlm.DlmError) as e:
        dlm.load_weights_mx(_cfg(), _weights(**{name: shape}))
    assert e.value.status == dlm.DLM_EINVAL and name in str(e.value)


def test_load_refuses_missing_buffers():
    for field in ("codes", "scales"):
        w = _weights()
        setattr(w.layers[1].w_o, field, None)
        with pytest.raises(dlm.DlmError) as e:
            dlm.load_weights_mx(_cfg(), w)
        assert "layer 1: w_o" in str(e.value)
    w = _weights()
    w.layers[0].ffn_norm = None
    with pytest.raises(dlm.DlmError):
        dlm.load_weights_mx(_cfg(), w)
    with pytest.raises(dlm.DlmError) as e:
        dlm.load_weights_mx(_cfg(head_dim=96), _weights())
    assert e.value.status == dlm.DLM_EUNSUPPORTED


class _Buf:
    def data_ptr(self):
        return FAKE


@pytest.fixture
def cache():
    m = dlm.load_weights_mx(_cfg(), _weights())
    _, need = dlm.kv_cache_alloc_mx(m, 3, 100)
    # per layer: codes and scales of keys and values, 3 slots x 2 heads x 128 positions
    assert need == 2 * 2 * (3 * 2 * 128 * 32 + 3 * 2 * 128 * 2)
    c, _ = dlm.kv_cache_alloc_mx(m, 3, 100, _Buf(), need)
    yield c
    dlm.cache_destroy(c)
    dlm.model_destroy(m)


@pytest.mark.parametrize("rows,layer,status", [
    ([(3, 10, 0, 1)], 0, dlm.DLM_EINVAL), ([(-1, 10, 0, 1)], 0, dlm.DLM_EINVAL),
    ([(0, 129, 0, 1)], 0, dlm.DLM_ESIZE), ([(0, -1, 0, 0)], 0, dlm.DLM_ESIZE),
    ([(0, 10, 0, -1)], 0, dlm.DLM_EINVAL), ([(0, 10, 8, 3)], 0, dlm.DLM_EINVAL),
    ([(0, 10, -1, 3)], 0, dlm.DLM_EINVAL), ([(0, 10, 2147483647, 2147483647)], 0, dlm.DLM_EINVAL),
    ([(0, 10, 0, 1)], 2, dlm.DLM_EINVAL), ([(0, 10, 0, 1)], -1, dlm.DLM_EINVAL),
    ([(0, 10, 0, 1), (0, 10, 4, 1)], 0, dlm.DLM_EINVAL), ([], 0, dlm.DLM_EINVAL),
    ([(0, 10, 0, 1)] * 65, 0, dlm.DLM_EINVAL),
])
def test_append_refused(cache, rows, layer, status):
    L = dlm.lib()
    r = dlm.make_kv_rows(rows)
    assert L.dlm_mx_kv_append(cache, layer, len(rows), r, FAKE, 1, FAKE, FAKE, None) == status
    if len(set(x[0] for x in rows)) == len(rows) or status != dlm.DLM_EINVAL:
        assert L.dlm_mx_kv_read(cache, layer, len(rows), r, FAKE, FAKE, None) == status


def test_cache_calls_refused(cache):
    L = dlm.lib()
    r = dlm.make_kv_rows([(1, 10, 0, 2)])
    E = dlm.DLM_EINVAL
    assert L.dlm_mx_kv_append(cache, 0, 1, r, FAKE, 0, FAKE, FAKE, None) == E
    for bad in (None, FAKE + 4):
        assert L.dlm_mx_kv_append(cache, 0, 1, r, bad, 1, FAKE, FAKE, None) == E
        assert L.dlm_mx_kv_append(cache, 0, 1, r, FAKE, 1, bad, FAKE, None) == E
        assert L.dlm_mx_kv_append(cache, 0, 1, r, FAKE, 1, FAKE, bad, None) == E
        assert L.dlm_mx_kv_read(cache, 0, 1, r, bad, FAKE, None) == E
        assert L.dlm_mx_kv_read(cache, 0, 1, r, FAKE, bad, None) == E
        assert L.dlm_mx_kv_attention(cache, 0, 1, r, bad, FAKE, None, 0, None) == E
        assert L.dlm_mx_kv_attention(cache, 0, 1, r, FAKE, bad, None, 0, None) == E
    assert L.dlm_mx_kv_append(None, 0, 1, r, FAKE, 1, FAKE, FAKE, None) == E
    assert L.dlm_mx_kv_append(cache, 0, 1, None, FAKE, 1, FAKE, FAKE, None) == E
    # no rows: nothing to do, no buffer is looked at
    r0 = dlm.make_kv_rows([(1, 0, 0, 0)])
    assert L.dlm_mx_kv_append(cache, 0, 1, r0, None, 1, None, None, None) == dlm.DLM_OK
    assert L.dlm_mx_kv_attention(cache, 0, 1, r0, None, None, None, 0, None) == dlm.DLM_OK
    assert dlm.mx_kv_attention_workspace(cache, r0) == 0


def test_attention_workspace_is_checked():
    m = dlm.load_weights_mx(_cfg(), _weights())
    _, need = dlm.kv_cache_alloc_mx(m, 1, 8192)
    c, _ = dlm.kv_cache_alloc_mx(m, 1, 8192, _Buf(), need)
    r = dlm.make_kv_rows([(0, 8192, 0, 4)])
    n = dlm.mx_kv_attention_workspace(c, r)
    assert n > 0      # few rows over a long cache: the keys are split
    L = dlm.lib()
    assert L.dlm_mx_kv_attention(c, 0, 1, r, FAKE, FAKE, None, n, None) == dlm.DLM_EINVAL
    assert L.dlm_mx_kv_attention(c, 0, 1, r, FAKE, FAKE, FAKE + 128, n, None) == dlm.DLM_EINVAL
    assert L.dlm_mx_kv_attention(c, 0, 1, r, FAKE, FAKE, FAKE, n - 1, None) == dlm.DLM_ESIZE
    dlm.cache_destroy(c)
    dlm.model_destroy(m)


def test_other_caches_are_refused():
    arr = (dlm.DlmLayerWeights * 2)(*[dlm.DlmLayerWeights(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE)] * 2)
    w = dlm.DlmWeights(FAKE, FAKE, FAKE, arr)
    m = dlm.load_weights(_cfg(), w)
    _, need = dlm.kv_cache_alloc(m, 2, 64)
    c, _ = dlm.kv_cache_alloc(m, 2, 64, _Buf(), need)
    r = dlm.make_kv_rows([(0, 10, 0, 1)])
    L = dlm.lib()
    assert L.dlm_mx_kv_append(c, 0, 1, r, FAKE, 1, FAKE, FAKE, None) == dlm.DLM_EUNSUPPORTED
    assert L.dlm_mx_kv_read(c, 0, 1, r, FAKE, FAKE, None) == dlm.DLM_EUNSUPPORTED
    assert L.dlm_mx_kv_attention(c, 0, 1, r, FAKE, FAKE, None, 0, None) == dlm.DLM_EUNSUPPORTED
    dlm.cache_destroy(c)
    dlm.model_destroy(m)


def test_binding_refuses_host_tensors_and_shapes():
    z = torch.zeros(4, 64, dtype=torch.bfloat16)
    q = _mx(8, 64)
    with pytest.raises(ValueError):
        dlm.mx_pack(torch.zeros(8, 64), q)            # not in device memory
    with pytest.raises(ValueError):
        dlm.mx_pack(torch.zeros(8, 63), q)            # another shape
    with pytest.raises(ValueError):
        dlm.mx_linear(z, q, torch.zeros(4, 8))
    with pytest.raises(ValueError):
        dlm.make_mx(torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 16, dtype=torch.uint8), 8, 64)
    with pytest.raises(ValueError):
        dlm.mx_linear_workspace(torch.float16, 4, q)


def test_binding_refuses_other_widths_and_types(cache):
    """What the model's heads and type do not fit is refused before its address is used."""
    r = dlm.make_kv_rows([(0, 10, 0, 2)])
    qkv, rot = torch.zeros(1, 2, 512), torch.zeros(2, 32, 2)
    q, k = torch.zeros(2, 256, dtype=torch.bfloat16), torch.zeros(2, 128, dtype=torch.bfloat16)
    for a in [(qkv[:, :, :511], rot, q), (qkv[:, :1], rot, q), (qkv, rot[:1], q), (qkv, rot[:, :31], q),
              (qkv, rot, q.float()), (qkv, rot, q[:, :255]), (qkv.double(), rot, q), (qkv, rot, q)]:
        with pytest.raises(ValueError):      # (the last one: not in device memory)
            dlm.mx_kv_append(cache, 0, r, *a)
    for a in [(k.float(), k), (k, k[:1]), (k[:, :64], k), (k, k)]:
        with pytest.raises(ValueError):
            dlm.mx_kv_read(cache, 0, r, *a)
    for a in [(q.float(), q), (q, q[:, ::2]), (q[:1], q), (q, q)]:
        with pytest.raises(ValueError):
            dlm.mx_kv_attention(cache, 0, r, *a)

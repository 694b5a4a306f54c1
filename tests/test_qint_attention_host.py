"""Steps of models in 8-bit integers leave their attention room for the key splits that it plans
(host only; the addresses below are never used)."""
import os

import pytest
import torch

from paper_2606_29094_amd import dlm

FAKE = 0x100000
HUGE = 1 << 40
pytestmark = pytest.mark.skipif(not os.path.exists(dlm.LIB_PATH), reason="libdlm.so not built")

# d_model, query heads, key/value heads, head_dim, d_ffn
SHAPES = {"mha": (4096, 32, 32, 128, 12288), "gqa": (3584, 28, 4, 128, 18944), "small": (256, 4, 2, 64, 688),
          "one group": (1024, 16, 1, 64, 2048)}


def _model(shape, int8, dtype=dlm.DLM_BF16):
    d, hq, hkv, dh, f = SHAPES[shape]
    cfg = dlm.DlmConfig(1, d, hq, hkv, dh, f, 2048, 2047, 1e-5, 1e4, 10.0, dtype)
    if not int8:
        w = dlm.DlmWeights(FAKE, FAKE, FAKE, (dlm.DlmLayerWeights * 1)(dlm.DlmLayerWeights(*[FAKE] * 6)))
        return dlm.load_weights(cfg, w)
    q = lambda n, k: dlm.DlmQint(FAKE, FAKE, n, k)
    layer = dlm.DlmLayerQint(FAKE, q((hq + 2 * hkv) * dh, d), q(d, hq * dh), FAKE, q(2 * f, d), q(d, f))
    return dlm.load_weights_qint(cfg, dlm.DlmWeightsQint(FAKE, FAKE, FAKE, (dlm.DlmLayerQint * 1)(layer)))


REQUESTS = [[n] for n in (1, 2, 5, 8, 12, 16, 17, 32, 63, 64, 96, 128, 129, 200, 256, 400, 512, 700)] + \
           [[1] * 3, [8] * 4, [32] * 2, [32] * 4, [64, 1, 17], [16] * 16]


@pytest.mark.parametrize("shape", SHAPES)
def test_splits_are_those_of_any_scratch(shape):
    _, hq, hkv, dh, _ = SHAPES[shape]
    for dtype, kind in ((dlm.DLM_BF16, torch.bfloat16), (dlm.DLM_F32, torch.float32)):
        model, dense = _model(shape, True, dtype), _model(shape, False, dtype)
        for rows in REQUESTS:
            room, other = (dlm.debug_attention_scratch(m, sum(rows), len(rows)) for m in (model, dense))
            for keys in (64, 300, 512, 1024, 2048, 8192):
                lens = [max(keys, n) for n in rows]
                if dtype == dlm.DLM_BF16:
                    plan = lambda b: dlm.debug_attention_plan(hq, hkv, dh, rows, lens, b)
                    assert plan(room) == plan(HUGE) and plan(room)[1] >= plan(other)[1], (rows, keys)
                plan = lambda b: dlm.debug_mx_attention_plan(kind, hq, hkv, dh, rows, lens, b)
                assert plan(room) == plan(HUGE), (rows, keys)
        dlm.model_destroy(model)
        dlm.model_destroy(dense)


def test_hook_refuses():
    m = _model("small", True)
    for rows, n_req in ((0, 1), (1, 0), (1, 65)):
        with pytest.raises(dlm.DlmError):
            dlm.debug_attention_scratch(m, rows, n_req)
    dlm.model_destroy(m)

"""The first kernel of a step of a model in 8-bit integers: the embedding's values exactly, in
rows that stay in registers and in wider ones; the first layer's norm is the operator's."""
import numpy as np
import pytest
import torch

from paper_2606_29094_amd import dlm, engine

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [128, 4096, 4160])
def test_first_layer_input(gpu, dtype, d):
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    V, dh, P, G = 64, 64, 21, 5
    g = torch.Generator().manual_seed(d)
    table = torch.randn(V, d, generator=g).to(dt).to(gpu)
    tok = np.random.default_rng(1).integers(0, V - 1, P).astype(np.int32)
    tok[3], tok[5] = -1, V                    # read as [MASK]
    one = (1 + torch.randn(d, generator=g) * 0.1).to(gpu)
    w = lambda r, c: (torch.randn(r, c, generator=g) * 0.1).to(dt).to(gpu)
    t = {"embed": table, "lm_head": w(V, d), "final_norm": one,
         "layers": [{"attn_norm": one, "w_qkv": w(3 * dh, d), "w_o": w(d, dh), "ffn_norm": one,
                     "w_gate_up": w(32, d), "w_down": w(d, 16)}]}
    model = engine.DeviceModel(engine.ModelShape(1, d, 1, 1, dh, 16, V, dtype), t, 1.0, int8=True)
    eng = engine.Engine(model, 1, P + G, "none")
    r = engine.Request(tok, G, G, 0.9)
    eng.admit(r, V - 1)
    out, _ = eng.debug_trace([r], 0, logits=False)
    ids = [v if 0 <= v < V else V - 1 for v in tok.tolist()] + [V - 1] * G
    rows = table[ids].float()
    assert torch.equal(out["h_in"], rows)
    n = len(ids)
    q = dlm.make_qint(torch.empty(dlm.qint_bytes(n, d)[0], dtype=torch.int8, device=gpu),
                      torch.empty(n, device=gpu), n, d)
    dlm.qint_norm(rows.contiguous(), one, 1e-5, q)
    want = torch.empty(n, d, dtype=dt, device=gpu)
    dlm.qint_unpack(q, want)
    assert torch.equal(out["a_attn"], want)

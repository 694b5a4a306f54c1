"""The packed model's step at row counts where its projections take the large tiles and the
unpacked way, with K slices left to the kernels that read them: every projection of a layer against
its 64-bit definition on the step's own inputs, and the logits next to those of the dense model of the same values."""
import dataclasses

import pytest
import torch

import mx_reference as ref
import synth
import synth.device as sdev
from helpers import logit_err
from paper_2606_29094_amd import dlm, engine
from test_gpu_mx_model import _requests, _shape, _unpacked

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
TILE64, TILE128, UNPACKED = 2, 3, 4

WIDE_FFN = dataclasses.replace(synth.GQA_7B, n_layers=2, d_model=2048, n_q_heads=14, n_kv_heads=2,
                               head_dim=128, d_ffn=4352, vocab=2048)
WIDE = dataclasses.replace(synth.GQA_7B, n_layers=2, d_model=4096, n_q_heads=16, n_kv_heads=2,
                           head_dim=128, d_ffn=2112, vocab=2048)
MODELS = {"ffn": WIDE_FFN, "wide": WIDE, "ffn-fp32": dataclasses.replace(WIDE_FFN, dtype="f32")}


def _plans(cfg, rows):
    dt, qd = (BF16 if cfg.dtype == "bf16" else F32), cfg.n_q_heads * cfg.head_dim
    plan = lambda n, k, **kw: dlm.debug_mx_linear_plan(dt, rows, n, k, **kw)[:2]
    return {"qkv": plan(qd + 2 * cfg.n_kv_heads * cfg.head_dim, cfg.d_model, join=False),
            "o": plan(cfg.d_model, qd, join=False),
            "gate_up": plan(2 * cfg.d_ffn, cfg.d_model, epilogue=dlm.DLM_MX_SWIGLU),
            "down": plan(cfg.d_model, cfg.d_ffn, join=False)}


@pytest.mark.parametrize("name,specs,plans", [
    ("ffn", [(500, 100, 0.9), (164, 100, 0.9)], {"gate_up": (TILE128, 1), "down": (TILE64, 2)}),
    ("wide", [(400, 100, 0.9), (36, 64, 0.9)], {"qkv": (TILE128, 4), "gate_up": (TILE64, 1)}),
    ("ffn", [(1200, 100, 0.9), (800, 100, 0.9)], {"gate_up": (UNPACKED, 1), "down": (UNPACKED, 2)}),
    ("wide", [(1200, 100, 0.9), (650, 100, 0.9)],
     {"qkv": (UNPACKED, 2), "o": (UNPACKED, 1), "gate_up": (UNPACKED, 1), "down": (UNPACKED, 1)}),
    ("ffn-fp32", [(400, 100, 0.9), (36, 64, 0.9)], {"gate_up": (TILE64, 1)})])
def test_projections_of_a_packed_step(gpu, name, specs, plans):
    cfg = MODELS[name]
    rows = sum(p + g for p, g, _ in specs)
    took = _plans(cfg, rows)
    assert {k: took[k] for k in plans} == plans
    t = sdev.model_tensors(cfg)
    packed = engine.DeviceModel(_shape(cfg), t, 10.0, packed=True)
    dense = engine.DeviceModel(_shape(cfg), _unpacked(packed, t, cfg), 10.0)
    dt = BF16 if cfg.dtype == "bf16" else F32
    z = []
    for model in (packed, dense):
        reqs = _requests(cfg, specs, 32)
        eng = engine.Engine(model, len(reqs), max(p + g for p, g, _ in specs), "dual")
        for r in reqs:
            eng.admit(r, cfg.mask_id)
        if model is packed:
            buf, splits = eng.debug_trace(reqs, 1, logits=False)
            assert splits == took["qkv"][1]
            for r in reqs:
                r.refreshed_block = -1
            b = {k: v.double() for k, v in buf.items()}
            w = {k: v.double() for k, v in dense.tensors["layers"][1].items()}

            def check(got, x, weight, base=None, slices=1):
                want, bound = x @ weight.T, ref.product_bound(x, weight, dt)
                if base is not None:      # the slices and the sum, added in fp32 one by one
                    bound = bound + ref.U * (slices + 1) * (base.abs() + x.abs() @ weight.abs().T)
                    want = want + base
                assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())

            qkv = b["qkv"].sum(0)
            check(qkv, b["a_attn"], w["w_qkv"])
            check(b["h_mid"], b["attn_out"], w["w_o"], b["h_in"], took["o"][1])
            check(b["h_out"], b["act"], w["w_down"], b["h_mid"], took["down"][1])
            p, bound = b["a_ffn"] @ w["w_gate_up"].T, ref.product_bound(b["a_ffn"], w["w_gate_up"], dt)
            (g, u), (tg, tu) = p.chunk(2, -1), bound.chunk(2, -1)
            err = (b["act"] - ref.silu_mul(g, u)).abs()
            assert bool((err <= ref.swiglu_bound(g, u, tg, tu, dt)).all())
        z.append(eng.debug_logits(reqs).cpu().numpy())
        eng.close()
    # (as in the smaller models' comparison: products differ in the order of their sums)
    assert logit_err(z[0], z[1]) < (2e-2 if dt == BF16 else 1e-4)

"""Models with projections in 8 bits: the step's path through the operators of test_gpu_qint."""
import dataclasses

import numpy as np
import pytest
import torch

import mx_reference
import synth
import synth.device as sdev
from paper_2606_29094_amd import dlm, engine

pytestmark = pytest.mark.gpu

GQA_SMALL = dataclasses.replace(synth.GQA_7B, n_layers=2, d_model=512, n_q_heads=14, n_kv_heads=2,
                                head_dim=64, d_ffn=1424, vocab=4096)
MHA_SMALL = dataclasses.replace(synth.MHA_8B, n_layers=2, d_model=1024, n_q_heads=8, n_kv_heads=8,
                                head_dim=128, d_ffn=2048, vocab=4096)
MODELS = {"tiny": synth.TINY_FP32, "gqa": GQA_SMALL, "mha": MHA_SMALL}
SPECS = [(100, 64, 0.9), (37, 50, 0.7), (64, 33, 0.95)]


def _model(cfg, inv_tau=10.0):
    return engine.DeviceModel(engine.ModelShape.of(cfg), sdev.model_tensors(cfg), inv_tau, int8=True)


def _requests(cfg, specs=SPECS, block=32):
    return [engine.Request(synth.tokens(30 + i, P, cfg.vocab), G, block, g)
            for i, (P, G, g) in enumerate(specs)]


def _start(cfg, model, mode, specs=SPECS, size=164, **kw):
    reqs = _requests(cfg, specs)
    eng = engine.Engine(model, len(specs), size, mode, **kw)
    for r in reqs:
        eng.admit(r, cfg.mask_id)
    return eng, reqs


def _packed(rows, k, dev):
    return dlm.make_qint(torch.empty(dlm.qint_bytes(rows, k)[0], dtype=torch.int8, device=dev),
                         torch.empty(rows, device=dev), rows, k)


def _values(q, dtype):
    out = torch.empty(q.n, q.k, dtype=dtype, device=q._keep[0].device)
    dlm.qint_unpack(q, out)
    return out


def _linear(x, w, epilogue, dtype, residual=None):
    y = torch.empty(x.n, w.n // 2 if epilogue == "swiglu" else w.n, dtype=dtype, device=x._keep[0].device)
    epi = dlm.QINT_EPILOGUES[epilogue]
    ws = torch.empty(max(1, dlm.qint_linear_workspace(x.n, w, epi)), dtype=torch.uint8, device=y.device)
    dlm.qint_linear(x, w, y, epi, ws, residual=residual)
    return y


def _check_layer(cfg, model, buf, layer, dt):
    """Each projection of a traced layer is the operator's on the values that it was given, bit
    for bit (a row's product does not depend on the others)."""
    l, n, dev = model.tensors["layers"][layer], buf["h_in"].shape[0], buf["h_in"].device
    x = _packed(n, cfg.d_model, dev)
    dlm.qint_norm(buf["h_in"], l["attn_norm"], model.shape.rms_eps, x)
    assert torch.equal(_values(x, dt), buf["a_attn"])
    assert torch.equal(_linear(x, l["w_qkv"], "store", torch.float32), buf["qkv"][0])
    a = _packed(n, buf["attn_out"].shape[1], dev)
    dlm.qint_pack(buf["attn_out"], a)
    assert torch.equal(_linear(a, l["w_o"], "add", torch.float32, buf["h_in"]), buf["h_mid"])
    dlm.qint_norm(buf["h_mid"], l["ffn_norm"], model.shape.rms_eps, x)
    assert torch.equal(_values(x, dt), buf["a_ffn"])
    assert torch.equal(_linear(x, l["w_gate_up"], "swiglu", dt), buf["act"])
    f = _packed(n, cfg.d_ffn, dev)
    dlm.qint_pack(buf["act"], f)
    assert torch.equal(_linear(f, l["w_down"], "add", torch.float32, buf["h_mid"]), buf["h_out"])


@pytest.mark.parametrize("name", list(MODELS))
@pytest.mark.parametrize("mode", ["none", "dual", "prefix"])
@pytest.mark.parametrize("packed_kv", [False, True])
def test_step_is_made_of_the_operators(gpu, name, mode, packed_kv):
    """Both layers of a recompute and of a cache step: the projections as above, attention
    against its definition on the step's queries and the stored keys and values, and each layer
    starts from what the one before left."""
    cfg = MODELS[name]
    model = _model(cfg)
    dt = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32
    hq, dh = cfg.n_q_heads, cfg.head_dim
    eng, reqs = _start(cfg, model, mode, packed_kv=packed_kv)
    for _ in range(2):
        ranges, last = eng.step_rows(reqs), None
        for layer in range(cfg.n_layers):
            saved = [r.refreshed_block for r in reqs]
            buf, splits = eng.debug_trace(reqs, layer)
            for r, s in zip(reqs, saved):
                r.refreshed_block = s
            assert splits == 1
            _check_layer(cfg, model, buf, layer, dt)
            assert last is None or torch.equal(last, buf["h_in"])
            last, at = buf["h_out"], 0
            for r, (r0, r1) in zip(reqs, ranges):
                m = r1 - r0
                k, v = (y.double() for y in eng.read_kv(layer, r.slot, r.seq_len))
                q = buf["q"][at:at + m].cpu().double().view(m, hq, dh)
                want, bound = mx_reference.attention(q, k, v, dt)
                err = (buf["attn_out"][at:at + m].cpu().double().view(m, hq, dh) - want).abs()
                assert bool((err <= bound).all()), float((err / bound).max())
                at += m
        eng.step(reqs)
    eng.close()


def test_steps_of_many_rows(gpu):
    """Rows for the large tiles, K slices among them, next to a request of a few."""
    cfg = dataclasses.replace(MHA_SMALL, n_layers=1, d_ffn=8192)
    model = _model(cfg)
    eng, reqs = _start(cfg, model, "dual", [(900, 64, 0.9), (700, 100, 0.9), (3, 9, 0.9)], 1024)
    assert dlm.debug_qint_linear_plan(1776, 1024, 8192)[1] > 1
    for _ in range(2):
        saved = [r.refreshed_block for r in reqs]
        buf, _ = eng.debug_trace(reqs, 0)
        for r, s in zip(reqs, saved):
            r.refreshed_block = s
        _check_layer(cfg, model, buf, 0, torch.bfloat16)
        eng.step(reqs)
    eng.close()


def test_gains_and_scales_at_any_address(gpu):
    """Gains and channel scales that start at no multiple of 16 bytes: the same steps."""
    cfg = dataclasses.replace(GQA_SMALL, d_ffn=4096)
    first = _model(cfg)

    def moved(t):
        big = torch.empty(t.numel() + 1, device=t.device)
        big[1:].copy_(t)
        return big[1:]

    def moved_scales(q):
        codes, scales = q._keep
        q2 = dlm.DlmQint(codes.data_ptr(), 0, q.n, q.k)
        q2._keep, q2._device = (codes, moved(scales)), q._device
        q2.scales = q2._keep[1].data_ptr()
        return q2

    layers = []
    for l in first.tensors["layers"]:
        l = {k: moved_scales(v) if isinstance(v, dlm.DlmQint) else v for k, v in l.items()}
        layers.append(dict(l, ffn_norm=moved(l["ffn_norm"])))
    second = engine.DeviceModel(first.shape, dict(first.tensors, layers=layers), 10.0, int8=True)
    assert dlm.debug_qint_linear_plan(96, cfg.d_model, cfg.d_ffn)[1] > 1      # (slices for the norm)
    outs = []
    for model in (first, second):
        eng, reqs = _start(cfg, model, "dual")
        for _ in range(3):
            eng.step(reqs)
        outs.append(eng.read_outputs(3))
        eng.close()
    for k in ("n", "block_conf", "block_tok"):
        assert np.array_equal(outs[0][k], outs[1][k]), k


@pytest.mark.parametrize("packed_kv", [False, True])
def test_generation_runs_and_repeats(gpu, packed_kv):
    """Whole generations: every position is unmasked, and a second run gives the same tokens."""
    cfg = GQA_SMALL
    model = _model(cfg)
    runs = []
    for _ in range(2):
        eng, reqs = _start(cfg, model, "dual", packed_kv=packed_kv)
        while any(not r.done for r in reqs):
            eng.step([r for r in reqs if not r.done])
        runs.append([eng.read_state(r) for r in reqs])
        eng.close()
    for (a, ma), (b, mb) in zip(*runs):
        assert not ma.any() and np.array_equal(a, b)


def test_step_without_allocation_and_matrices_packed_before(gpu):
    """dlm_denoise_step_noalloc, and a model over the 8-bit matrices of another."""
    cfg = GQA_SMALL
    first = _model(cfg)
    model = engine.DeviceModel(first.shape, first.tensors, 10.0, int8=True)
    assert model.tensors["layers"][0]["w_o"] is first.tensors["layers"][0]["w_o"]
    outs = []
    for noalloc in (False, True):
        eng, reqs = _start(cfg, model if noalloc else first, "dual")
        eng.step(reqs)
        if noalloc:
            batch = dlm.make_batch(eng.dlm_reqs(reqs), eng.tokens, eng.mask, eng.mode_id)
            dlm.denoise_step_noalloc(model.handle, eng.cache, batch, [r.threshold for r in reqs], eng.step_out)
        else:
            eng.enqueue_step(reqs)
        torch.cuda.synchronize()
        outs.append(eng.read_outputs(3))
        eng.close()
    for k in ("n", "block_conf", "block_tok"):
        assert np.array_equal(outs[0][k], outs[1][k]), k


@pytest.mark.parametrize("name", ["tiny", "gqa"])
def test_step_profile(gpu, name):
    """The profiler times every class of the step; a product of several kernels is one entry."""
    cfg = MODELS[name]
    model = _model(cfg)
    eng, reqs = _start(cfg, model, "dual")
    eng.step(reqs)
    dlm.profile_enable(model.handle, True)
    for _ in range(2):
        eng.step([r for r in reqs if not r.done])
    dlm.profile_enable(model.handle, False)
    prof = dlm.profile_read(model.handle)
    norms = [prof.get(kind, (0, 0, 0))[0] for kind in ("rmsnorm", "residual_rmsnorm")]
    assert sum(norms) == 2 * 2 * cfg.n_layers          # (the second adds a product's K slices)
    for kind, each in (("gemm_qkv", 1), ("rope_kv_write", 1), ("attention", 1),
                       ("pack_attention", 1), ("gemm_o", 1), ("gemm_gate_up_swiglu", 1), ("pack_act", 1),
                       ("gemm_down", 1)):
        calls, ms, seen = prof[kind]
        assert calls == seen == 2 * each * cfg.n_layers, kind
        assert 0 < ms < 1000, kind
    eng.close()

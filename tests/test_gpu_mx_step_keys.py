"""Keys that a step stores in a 4-bit cache: each within half a step of the rotated key, under the
scale that its group's largest magnitude gives."""
import pytest
import torch

import mx_reference as ref
import synth.device as sdev
from paper_2606_29094_amd import engine
from test_gpu_mx_model import MODELS, SPECS, _requests, _shape

pytestmark = pytest.mark.gpu


def _off_by(k, kr, delta):
    """How far k [g, 32] is from the nearest 4-bit values of kr, in units of what it may be: half a
    step and delta, under the scale of the group's largest magnitude (of either neighbour where
    delta reaches across a power of two)."""
    best = torch.full(k.shape[:1], float("inf"), dtype=torch.float64)
    top = kr.abs().amax(-1)
    for t in (top - delta.amax(-1), top, top + delta.amax(-1)):
        e = torch.ceil(torch.log2((t / 7).clamp_min(2.0 ** -126)))[:, None]
        y = kr.abs() / 2.0 ** e
        half = torch.where(y <= 2, 0.25, torch.where(y <= 4, 0.5, 1.0).double()) * 2.0 ** e
        ok = ((k - kr).abs() / (half + delta)).amax(-1)
        best = torch.minimum(best, ok)
    return best


@pytest.mark.parametrize("name", list(MODELS))
@pytest.mark.parametrize("mode", ["dual", "none"])
def test_stored_keys_are_the_rotated_ones(gpu, name, mode):
    cfg = MODELS[name]
    model = engine.DeviceModel(_shape(cfg), sdev.model_tensors(cfg), 10.0)
    hq, hkv, dh = cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim
    reqs = _requests(cfg, SPECS, 32)
    eng = engine.Engine(model, 3, 164, mode, packed_kv=True)
    for r in reqs:
        eng.admit(r, cfg.mask_id)
    for _ in range(2):
        ranges = eng.step_rows(reqs)
        saved = [r.refreshed_block for r in reqs]
        buf, splits = eng.debug_trace(reqs, 1, logits=False)
        for r, s in zip(reqs, saved):
            r.refreshed_block = s
        x = buf["qkv"].cpu()
        for s in range(1, splits):
            x[0] += x[s]
        x, at = x[0].view(-1, hq + 2 * hkv, dh)[:, hq:hq + hkv].double(), 0
        for r, (r0, r1) in zip(reqs, ranges):
            k = eng.read_kv(1, r.slot, r.seq_len)[0].double()[r0:r1]
            ang = torch.arange(r0, r1).double()[:, None] * \
                cfg.rope_theta ** (-torch.arange(dh // 2).double() / (dh // 2))
            a, b = x[at:at + r1 - r0].chunk(2, -1)
            c, s = ang.cos()[:, None], ang.sin()[:, None]
            kr = torch.cat([a * c - b * s, b * c + a * s], -1)
            # cosine and sine, two products and their sum, each rounded to fp32
            delta = 3 * ref.U * torch.cat([a.abs() + b.abs()] * 2, -1)
            off = _off_by(*(t.reshape(-1, 32) for t in (k, kr, delta)))
            assert bool((off <= 1).all()), float(off.max())
            at += r1 - r0
        eng.step(reqs)
    eng.close()

"""The operators on 4-bit operands: packing, products, and a key/value cache in 4 bits.

A 4-bit matrix is a row of groups of 32 consecutive values: a byte e for each group
(its scale 2^(e - 127)) and a 4-bit code for each value, sign and one of 0, 0.5, 1, 1.5,
2, 3, 4, 6, even elements in the low halves of the bytes. Each case is one call (a
cache append: the call and the read-back of what it stored) at the layer shapes of the
repository's models, or of generic ones.
"""
import functools
import math
import random

import numpy as np
import torch

own = False

GROUP = 32
# head layouts and storage types of the repository's models, and generic ones
HEADS = {
    "mha-8b": dict(hq=32, hkv=32, dh=128, dtype="bf16"),
    "gqa-7b": dict(hq=28, hkv=4, dh=128, dtype="bf16"),
    "tiny-fp32": dict(hq=4, hkv=4, dh=64, dtype="f32"),
    "gqa-64": dict(hq=12, hkv=2, dh=64, dtype="bf16"),
    "gqa-fp32": dict(hq=8, hkv=2, dh=128, dtype="f32"),
}
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
MAX_PRODUCT = 1000 * 37888 * 3584      # rows x outputs x inputs of the largest product
MAX_SCORES = 8 * 32 * 1280 * 1280      # rows x heads x keys of the largest attention


def _linear(name, rows, n, k, epilogue="store", dtype="bf16", pad=0):
    return {"name": name, "kind": "linear", "rows": rows, "n": n, "k": k, "epilogue": epilogue,
            "dtype": dtype, "pad": pad}


def _pack(name, n, k, dtype="bf16"):
    return {"name": name, "kind": "pack", "n": n, "k": k, "dtype": dtype}


def _cache(name, kind, heads, batch, prompt, gen, block, refresh=0, splits=1, mix=0):
    return {"name": name, "kind": kind, "heads": heads, "batch": batch, "prompt_lo": prompt[0],
            "prompt_hi": prompt[1], "gen": gen, "block": block, "refresh": refresh,
            "splits": splits, "mix": mix}


def listed():
    return [
        # output projection of a single row: the smallest call, latency
        _linear("linear-o-1", 1, 4096, 4096),
        # gate/up of one request's block of 32: weights streamed once
        _linear("linear-gate-up-32", 32, 24576, 4096, "swiglu"),
        # down projection of one request's block of 64 into the residual stream
        _linear("linear-down-64", 64, 3584, 18944, "add"),
        # the fp32 model's type at sizes that fit no tile
        _linear("linear-odd-fp32", 37, 689, 1031, dtype="f32"),
        # gate/up of a recompute step: bound by the matrix cores
        _linear("linear-gate-up-1000", 1000, 37888, 3584, "swiglu"),
        # one output projection packed while a model is loaded
        _pack("pack-o", 4096, 4096),
        # a gate/up matrix held in fp32
        _pack("pack-gate-up-fp32", 37888, 3584, "f32"),
        # keys and values of one user's block of 32, from a product in two K slices
        _cache("append-mha-b1", "append", "mha-8b", 1, (261, 261), 256, 32, splits=2),
        # a batch of 8 recomputed whole: 10240 rows
        _cache("append-refresh-b8", "append", "mha-8b", 8, (1024, 1024), 256, 32, refresh=8),
        # one user decoding with a dual cache
        _cache("attn-mha-b1", "attn", "mha-8b", 1, (261, 261), 256, 32),
        # the default benchmark's batch of 64: 4096 rows of 28 heads over 4 cached ones
        _cache("attn-gqa-b64", "attn", "gqa-7b", 64, (512, 512), 512, 64, mix=2),
        # a batch of 8 recomputed whole
        _cache("attn-refresh-b8", "attn", "mha-8b", 8, (1024, 1024), 256, 32, refresh=8),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.choice(["linear", "linear", "linear", "pack", "append", "attn", "attn"])
    if kind in ("linear", "pack"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        n, k = rng.choice([(4096, 4096), (12288, 4096), (24576, 4096), (4096, 12288), (4608, 3584),
                           (3584, 18944), (37888, 3584), (1376, 256), (256, 688),
                           (log(1, 20000), log(1, 20000)), (log(1, 20000), 8 * log(1, 2500))])
        if kind == "pack":
            c = _pack("", n, k, dtype)
        else:
            c = _linear("", log(1, 4096), n, k, rng.choice(["store", "add", "swiglu"]), dtype,
                        rng.choice([0, 0, 0, 8, 3]))
            c["n"] += c["n"] % 2 if c["epilogue"] == "swiglu" else 0
            cap = MAX_PRODUCT // (1 if dtype == "bf16" else 8)
            while c["rows"] * c["n"] * c["k"] > cap:
                c["rows"] = (c["rows"] + 1) // 2
    else:
        lo = log(1, 1500)
        c = _cache("", kind, rng.choice(list(HEADS)), log(1, 64),
                   (lo, min(4096, int(lo * rng.uniform(1, 4)) + 1)), log(1, 1024),
                   rng.choice([1, 16, 24, 32, 32, 57, 64, 64]), mix=rng.randrange(1 << 20))
        if kind == "append":
            c["splits"] = rng.choice([1, 1, 2, 4])
        if rng.random() < 0.4:
            c["refresh"] = rng.randint(1, c["batch"])
        while _cost(c) > 1:
            c["batch"] = (c["batch"] + 1) // 2
            c["refresh"] = min(c["refresh"], c["batch"])
            if c["batch"] == 1:
                c["prompt_lo"], c["prompt_hi"] = c["prompt_lo"] // 2 + 1, c["prompt_hi"] // 2 + 1
    del c["name"]
    return c


# ------------------------------------------------------------------ shapes
def _groups(k):
    return -(-k // GROUP)


def _scale_ld(k):
    return -(-_groups(k) // 16) * 16


def _requests(case):
    """(sequence length, first row's position, rows) of each request: the first ``refresh``
    recompute their whole sequence, the others one block."""
    r = random.Random(case["mix"])
    out = []
    for i in range(case["batch"]):
        p = r.randint(case["prompt_lo"], case["prompt_hi"])
        k = r.randrange(-(-case["gen"] // case["block"]))
        s = p + k * case["block"]
        n = min(case["block"], p + case["gen"] - s)
        out.append((p + case["gen"], 0, p + case["gen"]) if i < case["refresh"]
                   else (p + case["gen"], s, n))
    return out


def _cost(case):
    """The call's work over that of the largest one of its kind."""
    h, reqs = HEADS[case["heads"]], _requests(case)
    size = SIZE[h["dtype"]] // 2
    rows = sum(n for _, _, n in reqs)
    if case["kind"] == "append":
        return rows * (h["hq"] + 2 * h["hkv"]) * h["dh"] * case["splits"] / (10240 * 96 * 128)
    # what the plain form pads the batch to, and what each side computes
    padded = len(reqs) * max(n for _, _, n in reqs) * max(l for l, _, _ in reqs) * h["hq"]
    return max(size ** 3 * sum(n * l for l, _, n in reqs) * h["hq"] / MAX_SCORES,
               padded / (4 * MAX_SCORES))


def work(case):
    if case["kind"] in ("linear", "pack"):
        n, k, es = case["n"], case["k"], SIZE[case["dtype"]]
        packed = n * _groups(k) * 17
        if case["kind"] == "pack":             # read; pack; the values read back
            return {"bytes": 2 * n * k * es + 2 * packed, "flops": 4 * n * k}
        m, out = case["rows"], {"store": 4 * n, "add": 8 * n, "swiglu": n // 2 * es}[case["epilogue"]]
        return {"bytes": packed + m * k * es + m * out, "flops": 2 * m * n * k}
    h, reqs = HEADS[case["heads"]], _requests(case)
    es, rows = SIZE[h["dtype"]], sum(n for _, _, n in reqs)
    head = _groups(h["dh"]) * 17               # bytes of one cached head vector
    if case["kind"] == "append":
        qkv = (h["hq"] + 2 * h["hkv"]) * h["dh"]
        return {"bytes": rows * (case["splits"] * qkv * 4 + h["dh"] * 4 + h["hq"] * h["dh"] * es +
                                 4 * h["hkv"] * head + 2 * h["hkv"] * h["dh"] * es),
                "flops": rows * qkv * (case["splits"] + 6)}
    return {"bytes": sum(l for l, _, _ in reqs) * 2 * h["hkv"] * head + 2 * rows * h["hq"] * h["dh"] * es,
            "flops": 4 * sum(n * l for l, _, n in reqs) * h["hq"] * h["dh"]}


# ------------------------------------------------------------- 4-bit groups
def _values(codes, scales, k):
    """The values [n, k] (fp32) of codes [n, 16 G] and scales [n, >= G]."""
    g = codes.shape[1] // 16
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    table = torch.cat([table, -table])
    nib = torch.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], g, GROUP)
    e = scales[:, :g].to(torch.int32)
    s = (e << 23).view(torch.float32)
    s = torch.where(e == 255, torch.full_like(s, math.nan), s)
    return (table[nib.long()] * s[..., None]).reshape(codes.shape[0], g * GROUP)[:, :k]


def _encode(w):
    """codes [n, 16 G] and scales [n, padded G] of w [n, k] (fp32)."""
    n, k = w.shape
    g = _groups(k)
    x = torch.nn.functional.pad(w, (0, g * GROUP - k)).reshape(n, g, GROUP)
    amax = x.abs().amax(-1)
    bits = amax.view(torch.int32)
    e = ((bits >> 23) - 2 + ((bits & 0x7fffff) > 0x600000).int()).clamp(2, 252)
    y = x.abs() * ((254 - e) << 23).view(torch.float32)[..., None]
    code = ((y > .25).to(torch.uint8) + (y >= .75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) +
            (y >= 3.5) + (y > 5)).to(torch.uint8) | (torch.signbit(x).to(torch.uint8) << 3)
    bad = ~torch.isfinite(amax)
    code = torch.where(bad[..., None], torch.zeros_like(code), code)
    e = torch.where(bad, torch.full_like(e, 255), e)
    code = code.reshape(n, g * 16, 2)
    codes = code[..., 0] | (code[..., 1] << 4)
    return codes, torch.nn.functional.pad(e.to(torch.uint8), (0, _scale_ld(k) - g))


# ------------------------------------------------------------------ inputs
def _normal(gen, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["kind"] in ("linear", "pack"):
        n, k, dt = case["n"], case["k"], DTYPE[case["dtype"]]
        w = _normal(gen, n, k, std=0.02, dtype=dt)
        if case["kind"] == "pack":
            s["w"] = w
            if own:
                from paper_2606_29094_amd import dlm
                s["codes"] = torch.empty(n, 16 * _groups(k), dtype=torch.uint8, device="cuda")
                s["scales"] = torch.empty(n, _scale_ld(k), dtype=torch.uint8, device="cuda")
                s["out"] = torch.empty(n, k, dtype=dt, device="cuda")
                s["mx"] = dlm.make_mx(s["codes"], s["scales"], n, k)
            return s
        s["codes"], s["scales"] = _encode(w.float())
        m = case["rows"]
        x = _normal(gen, m, k + case["pad"])
        if case["epilogue"] == "add":            # a gated activation
            x = x * _normal(gen, m, k + case["pad"])
        s["x"] = x.to(dt)[:, :k]
        out = {"store": (m, n), "add": (m, n), "swiglu": (m, n // 2)}[case["epilogue"]]
        if case["epilogue"] == "add":
            s["h"] = _normal(gen, m, n)
        if own:
            from paper_2606_29094_amd import dlm
            s["y"] = torch.empty(out, dtype=dt if case["epilogue"] == "swiglu" else torch.float32,
                                 device="cuda")
            s["mx"] = dlm.make_mx(s["codes"], s["scales"], n, k)
            s["epilogue"] = dlm.MX_EPILOGUES[case["epilogue"]]
            s["ws"] = torch.empty(max(1, dlm.mx_linear_workspace(dt, m, s["mx"], s["epilogue"])),
                                  dtype=torch.uint8, device="cuda")
        return s
    h, reqs = HEADS[case["heads"]], _requests(case)
    hq, hkv, dh, dt = h["hq"], h["hkv"], h["dh"], DTYPE[h["dtype"]]
    rows, longest = sum(n for _, _, n in reqs), max(l for l, _, _ in reqs)
    slots, s_max = case["batch"], -(-longest // 64) * 64
    # request i's cache is in slot (i * 5 + 2) mod batch or, where that repeats, in its own
    slot = [(i * 5 + 2) % slots if slots % 5 else i for i in range(slots)]
    row0 = np.cumsum([0] + [n for _, _, n in reqs])
    s["slot"] = torch.tensor(slot, device="cuda")
    s["len"] = torch.tensor([l for l, _, _ in reqs], device="cuda")
    s["rows"] = torch.tensor([n for _, _, n in reqs], device="cuda")
    s["row0"] = torch.tensor(row0[:-1].copy(), device="cuda")
    s["longest"], s["most"] = longest, max(n for _, _, n in reqs)
    per = slots * hkv * s_max
    if case["kind"] == "append":
        pos = torch.cat([torch.arange(p, p + n, dtype=torch.float64, device="cuda") for _, p, n in reqs])
        freq = 10000.0 ** (-torch.arange(dh // 2, dtype=torch.float64, device="cuda") / (dh // 2))
        ang = pos[:, None] * freq
        s["rot"] = torch.stack([ang.cos(), ang.sin()], -1).float()
        s["qkv"] = _normal(gen, case["splits"], rows, (hq + 2 * hkv) * dh, std=case["splits"] ** -0.5)
    else:
        s["q"] = _normal(gen, rows, hq * dh, std=1.5, dtype=dt)
        kv = [_encode(_normal(gen, per, dh)) for _ in range(2)]
        g = dh // GROUP
        # positions behind a sequence hold whatever was there before: not even numbers
        pos = torch.arange(s_max, device="cuda")
        limit = torch.zeros(slots, dtype=torch.long, device="cuda").index_copy(0, s["slot"], s["len"])
        behind = (pos[None] >= limit[:, None])[:, None, :, None].expand(slots, hkv, s_max, g)
        sc = [e[:, :g].reshape(slots, hkv, s_max, g).masked_fill(behind, 255).contiguous() for _, e in kv]
        s["kc"], s["vc"] = (c.reshape(slots, hkv, s_max, dh // 2) for c, _ in kv)
        s["ks"], s["vs"] = sc
    if own:
        from paper_2606_29094_amd import dlm, engine
        # one layer of a model with these heads
        d, f, v = 64, 64, 64
        z = lambda *shape, dtype=dt: torch.zeros(*shape, dtype=dtype, device="cuda")
        shape = engine.ModelShape(1, d, hq, hkv, dh, f, v, h["dtype"])
        layer = {"attn_norm": z(d, dtype=torch.float32), "w_qkv": z(shape.qkv_dim, d),
                 "w_o": z(d, hq * dh), "ffn_norm": z(d, dtype=torch.float32),
                 "w_gate_up": z(2 * f, d), "w_down": z(d, f)}
        s["model"] = engine.DeviceModel(shape, {"embed": z(v, d), "lm_head": z(v, d),
                                                "final_norm": z(d, dtype=torch.float32),
                                                "layers": [layer]}, 1.0)
        _, need = dlm.kv_cache_alloc_mx(s["model"].handle, slots, s_max)
        s["buf"] = torch.zeros(need, dtype=torch.uint8, device="cuda")
        s["cache"], _ = dlm.kv_cache_alloc_mx(s["model"].handle, slots, s_max, s["buf"], need)
        s["kv_rows"] = dlm.make_kv_rows([(slot[i], l, p, n) for i, (l, p, n) in enumerate(reqs)])
        if case["kind"] == "append":
            s["out"] = {"q": torch.empty(rows, hq * dh, dtype=dt, device="cuda"),
                        "k": torch.empty(rows, hkv * dh, dtype=dt, device="cuda"),
                        "v": torch.empty(rows, hkv * dh, dtype=dt, device="cuda")}
        else:
            # key codes, value codes, key scales, value scales of the layer
            parts = [x.reshape(-1) for x in (s["kc"], s["vc"], s["ks"], s["vs"])]
            at = 0
            for x in parts:
                s["buf"][at:at + x.numel()].copy_(x)
                at += -(-x.numel() // 256) * 256
            s["out"] = torch.empty(rows, hq * dh, dtype=dt, device="cuda")
            s["ws"] = torch.empty(max(1, dlm.mx_kv_attention_workspace(s["cache"], s["kv_rows"])),
                                  dtype=torch.uint8, device="cuda")
    return s


# -------------------------------------------------------------------- runs
def run(s):
    case = s["case"]
    return {"linear": _run_linear, "pack": _run_pack, "append": _run_append,
            "attn": _run_attn}[case["kind"]](s, case)


def _run_pack(s, case):
    if own:
        from paper_2606_29094_amd import dlm
        dlm.mx_pack(s["w"], s["mx"])
        dlm.mx_unpack(s["mx"], s["out"])
        return s["out"]
    return _values(*_encode(s["w"].float()), case["k"]).to(s["w"].dtype)


def _run_linear(s, case):
    if own:
        from paper_2606_29094_amd import dlm
        if case["epilogue"] == "add":
            s["y"].copy_(s["h"])
        dlm.mx_linear(s["x"], s["mx"], s["y"], s["epilogue"], s["ws"])
        return s["y"]
    y = s["x"].float() @ _values(s["codes"], s["scales"], case["k"]).T
    if case["epilogue"] == "add":
        return s["h"] + y
    if case["epilogue"] == "swiglu":
        gate, up = y.chunk(2, -1)
        return (gate / (1 + torch.exp(-gate)) * up).to(s["x"].dtype)
    return y


def _rotate(x, rot):
    """x [N, heads, dh], rot [N, dh / 2, 2]: pairs (i, i + dh / 2) turned by their angle."""
    a, b = x.chunk(2, -1)
    c, d = rot[:, None, :, 0], rot[:, None, :, 1]
    return torch.cat([a * c - b * d, b * c + a * d], -1)


def _run_append(s, case):
    if own:
        from paper_2606_29094_amd import dlm
        o = s["out"]
        dlm.mx_kv_append(s["cache"], 0, s["kv_rows"], s["qkv"], s["rot"], o["q"])
        dlm.mx_kv_read(s["cache"], 0, s["kv_rows"], o["k"], o["v"])
        return o
    h = HEADS[case["heads"]]
    hq, hkv, dh, dt = h["hq"], h["hkv"], h["dh"], DTYPE[h["dtype"]]
    x = functools.reduce(torch.add, s["qkv"].unbind(0))      # slices in order
    x = x.reshape(x.shape[0], hq + 2 * hkv, dh)
    q, k, v = x.split([hq, hkv, hkv], 1)
    back = lambda t: _values(*_encode(t.reshape(-1, dh)), dh).reshape(-1, hkv * dh).to(dt)
    return {"q": _rotate(q, s["rot"]).reshape(-1, hq * dh).to(dt), "k": back(_rotate(k, s["rot"])),
            "v": back(v)}


def _run_attn(s, case):
    if own:
        from paper_2606_29094_amd import dlm
        dlm.mx_kv_attention(s["cache"], 0, s["kv_rows"], s["q"], s["out"], s["ws"])
        return s["out"]
    return _attention(s, case, torch.float32).to(s["q"].dtype)


def _attention(s, case, dt):
    """Softmax attention of every row over the cached positions of its request."""
    h = HEADS[case["heads"]]
    hq, hkv, dh = h["hq"], h["hkv"], h["dh"]
    R, S, n = len(s["slot"]), s["longest"], s["most"]

    def cached(codes, scales):
        c = codes[:, :, :S].index_select(0, s["slot"]).reshape(-1, dh // 2)
        e = scales[:, :, :S].index_select(0, s["slot"]).reshape(-1, dh // GROUP)
        x = _values(c, e, dh).reshape(R, hkv, S, dh)
        seen = torch.arange(S, device=x.device)[None] < s["len"][:, None]
        return x.masked_fill(~seen[:, None, :, None], 0).to(dt), seen

    k, seen = cached(s["kc"], s["ks"])
    v, _ = cached(s["vc"], s["vs"])
    i = torch.arange(n, device=k.device)
    at = s["row0"][:, None] + torch.minimum(i[None], s["rows"][:, None] - 1)     # rows padded per request
    q = s["q"].to(dt)[at].reshape(R, n, hkv, hq // hkv, dh).permute(0, 2, 3, 1, 4).reshape(R, hkv, -1, dh)
    z = torch.matmul(q, k.transpose(2, 3).contiguous()) * dh ** -0.5
    z = z.masked_fill_(~seen[:, None, None, :], -math.inf)
    z = torch.exp(z.sub_(z.amax(-1, keepdim=True)))
    o = torch.matmul(z, v) / z.sum(-1, keepdim=True)
    o = o.reshape(R, hkv, hq // hkv, n, dh).permute(0, 3, 1, 2, 4).reshape(R, n, hq * dh)
    return o[i[None] < s["rows"][:, None]]


# ------------------------------------------------------------------- exact
def _exact_values(codes, scales, k):
    """The same values in 64 bits, from sign, exponent and mantissa of each code."""
    c = codes.long()
    nib = torch.empty(c.shape[0], 2 * c.shape[1], dtype=torch.long, device=c.device)
    nib[:, 0::2], nib[:, 1::2] = c % 16, c // 16
    sign, ex, man = 1.0 - 2.0 * (nib // 8).double(), (nib % 8) // 2, (nib % 2).double()
    mag = torch.where(ex == 0, man / 2, (1 + man / 2) * 2.0 ** (ex - 1).double())
    e = scales[:, :c.shape[1] // 16].double().repeat_interleave(GROUP, 1)
    return (sign * mag * torch.exp2(e - 127))[:, :k]


def _exact_round(w):
    """w [n, k] (64 bits) in groups of 32 at the nearest representable value, ties to the
    even code; the group's largest magnitude lies within (3.5, 7] scales."""
    n, k = w.shape
    g = _groups(k)
    x = torch.zeros(n, g * GROUP, dtype=torch.float64, device=w.device)
    x[:, :k] = w
    x = x.reshape(n, g, GROUP)
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(amax.clamp_min(2.0 ** -140) / 7)).clamp(-125, 125)
    y = x.abs() / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.clamp_min(1.0))).clamp_max(2.0) - 1)
    q = (torch.round(y / step) * step).clamp_max(6.0)
    return (torch.sign(x) * q * torch.exp2(e)).reshape(n, -1)[:, :k]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "pack":
        return _exact_round(s["w"].double())
    if case["kind"] == "linear":
        y = s["x"].double() @ _exact_values(s["codes"], s["scales"], case["k"]).T
        if case["epilogue"] == "add":
            return s["h"].double() + y
        if case["epilogue"] == "swiglu":
            gate, up = y[:, :case["n"] // 2], y[:, case["n"] // 2:]
            return gate * torch.sigmoid(gate) * up
        return y
    h, reqs = HEADS[case["heads"]], _requests(case)
    hq, hkv, dh = h["hq"], h["hkv"], h["dh"]
    if case["kind"] == "append":
        x = s["qkv"].double().sum(0)
        cos, sin = s["rot"].double()[..., 0], s["rot"].double()[..., 1]
        z = torch.complex(cos, sin)[:, None]
        turn = lambda t: (lambda u: torch.cat([u.real, u.imag], -1))(
            torch.complex(t[..., :dh // 2].contiguous(), t[..., dh // 2:].contiguous()) * z)
        heads = lambda a, b: x[:, a * dh:b * dh].reshape(-1, b - a, dh)
        # the stored keys and values are whole steps apart: what is exact there is the
        # rounding of the 32-bit sums, which the plain form defines
        return {"q": turn(heads(0, hq)).reshape(-1, hq * dh), "k": None, "v": None}
    out, at = [], 0
    for i, (l, _, n) in enumerate(reqs):       # request by request, head by head
        slot = int(s["slot"][i])
        q = s["q"][at:at + n].double().reshape(n, hq, dh)
        at += n
        o = torch.empty(n, hq, dh, dtype=torch.float64, device=q.device)
        for j in range(hkv):
            k = _exact_values(s["kc"][slot, j, :l], s["ks"][slot, j, :l], dh)
            v = _exact_values(s["vc"][slot, j, :l], s["vs"][slot, j, :l], dh)
            a, b = j * (hq // hkv), (j + 1) * (hq // hkv)
            z = q[:, a:b].permute(1, 0, 2).reshape(-1, dh) @ k.T / math.sqrt(dh)
            o[:, a:b] = (torch.softmax(z, -1) @ v).reshape(b - a, n, dh).permute(1, 0, 2)
        out.append(o.reshape(n, hq * dh))
    return torch.cat(out)

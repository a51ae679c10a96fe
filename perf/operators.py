"""The quantized linear layer's surroundings in a transformer block, as cases that can be timed.

A case is one pass through an operator of paper_2412_19867_amd.wq.LinearPlan with everything a program
keeps between passes (plan, prepared weights, workspace, output buffers) in hand:

  norm      LinearPlan.rms_norm_quantize   h = x + residual, root-mean-square norm of h, group-wise int8
                                           codes and scales of it; h itself is an output too
  quantize  LinearPlan.quantize_rows       group-wise int8 codes and scales of rows of any float type
  linear    LinearPlan.linear              rows quantized, multiplied with W8A8 or W4A8 weights, bias,
                                           activation (gated or not) and residual
  block     the three in turn              norm -> gated product -> product with residual

Plain forms (`own` false) compute the same from elementary torch operations in fp32.  The int8 codes
are whole numbers that both sides have to agree on, so what decides a code is defined to the last
bit: a group's scale is fl(a / 127), a code rint(fl(v fl(127 / a))), the norm's factor
fl(1 / sqrt(mean + eps)) of a sum of squares in 64 bits (which no order of summation changes).
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}
TINY = 2.0 ** -126   # the smallest normal fp32 number
EPS = 1e-6


def _norm(name, rows, C, g, dtype, residual=True):
    return {"name": name, "kind": "norm", "rows": rows, "Cin": C, "g": g, "dtype": dtype, "residual": residual}


def _linear(name, rows, Cin, Cout, g, bits, dtype, act="none", gated=False, residual=False):
    return {"name": name, "kind": "linear", "rows": rows, "Cin": Cin, "Cout": Cout, "g": g, "bits": bits,
            "dtype": dtype, "act": act, "gated": gated, "residual": residual}


def listed():
    return [
        # decoding one token: latency of one small launch
        _norm("norm_1x4096", 1, 4096, 128, "bf16"),
        # a prompt's tokens in a wide model, half precision, no residual yet (the first layer of a block)
        _norm("norm_777x5120", 777, 5120, 32, "fp16", residual=False),
        # a large batch of tokens with the residual stream in fp32
        _norm("norm_4096x8192_fp32", 4096, 8192, 64, "fp32"),
        # the attention's output of an image's tokens in front of its projection
        {"name": "quantize_4096x1280", "kind": "quantize", "rows": 4096, "Cin": 1280, "g": 64, "dtype": "bf16"},
        # as many rows as a serving batch has, odd in number, one group a lane's width
        {"name": "quantize_33x640", "kind": "quantize", "rows": 33, "Cin": 640, "g": 32, "dtype": "fp32"},
        # decoding one token: the down projection with its residual, 4-bit weights are all that is read
        _linear("token_8192_4096_w4", 1, 8192, 4096, 128, 4, "bf16", residual=True),
        # a few tokens at once: the wide gated projection, 8-bit weights
        _linear("batch16_gated_4096", 16, 4096, 2 * 8192, 128, 8, "bf16", "silu", gated=True),
        # a text encoder's feed-forward layer: 77 tokens, nothing fills a tile
        _linear("encoder_77x768", 77, 768, 2048, 32, 8, "fp16", "gelu_tanh"),
        # a diffusion transformer's gated feed-forward layer over an image's tokens, fp32
        _linear("image_gated_1280", 4096, 1280, 2 * 5120, 64, 8, "fp32", "gelu", gated=True),
        # an odd number of a prompt's tokens through an output projection that no tile divides
        _linear("prompt_1001x2048", 1001, 2048, 2040, 256, 4, "bf16", residual=True),
        # the largest product: a long prompt through a wide gated projection
        _linear("prompt_gated_4096", 4096, 4096, 2 * 8192, 128, 4, "bf16", "silu", gated=True),
        # a whole feed-forward block over a batch of tokens
        {"name": "block_512x4096", "kind": "block", "rows": 512, "Cin": 4096, "width": 8192, "g": 128, "bits": 4,
         "dtype": "bf16"},
    ]


# ---- drawn cases ----

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _channels(rng, lo, hi, step):
    return max(step, (_log(rng, lo, hi) + step // 2) // step * step)


def draw(rng):
    while True:
        kind = rng.choices(("norm", "quantize", "linear", "block"), (25, 10, 55, 10))[0]
        g, dtype = rng.choice((32, 64, 64, 128, 128, 256, 512)), rng.choice(("bf16", "bf16", "fp16", "fp32"))
        if kind == "norm":
            c = _norm(None, _log(rng, 1, 8192), _channels(rng, 320, 16384, g), g, dtype, rng.random() < 0.75)
        elif kind == "quantize":
            c = {"kind": kind, "rows": _log(rng, 1, 8192), "Cin": _channels(rng, 320, 16384, g), "g": g, "dtype": dtype}
        elif kind == "linear":
            gated = rng.random() < 0.35
            if gated:
                out = 2 * _channels(rng, 320, 8192, 16)
            else:   # mostly multiples of 32, sometimes any number
                out = _log(rng, 320, 16384) if rng.random() < 0.25 else _channels(rng, 320, 16384, 32)
            c = _linear(None, _log(rng, 1, 8192), _channels(rng, 320, 8192, g), out, g, rng.choice((8, 4)), dtype,
                        rng.choice(("none", "relu", "silu", "gelu", "gelu_tanh")), gated, rng.random() < 0.5)
        else:
            c = {"kind": kind, "rows": _log(rng, 1, 2048), "Cin": _channels(rng, 320, 4096, g),
                 "width": _channels(rng, 640, 8192, g), "g": g, "bits": rng.choice((8, 4)), "dtype": rng.choice(("bf16", "fp16"))}
        c.pop("name", None)
        w = work(c)
        if w["bytes"] <= 440e6 and w["flops"] <= 560e9:
            return c


# ---- what a case needs ----

def _linear_work(rows, Cin, Cout, outs, g, bits, e, residual, codes=False):
    return (rows * (Cin + 4 * Cin / g if codes else e * Cin) + Cout * (Cin * bits / 8 + 4 * (Cin // g) + 4) +
            e * rows * outs * (2 if residual else 1), 2 * rows * Cin * Cout)


def work(case):
    c, e = case, SIZES[case["dtype"]]
    if c["kind"] in ("norm", "quantize"):
        n, norm = c["rows"] * c["Cin"], c["kind"] == "norm"
        b = n * (e + 1 + 4 / c["g"]) + (n * e * (2 if c["residual"] else 1) + 4 * c["Cin"] if norm else 0)
        f = n * (8 if norm else 4)
    elif c["kind"] == "linear":
        outs = c["Cout"] // 2 if c["gated"] else c["Cout"]
        b, f = _linear_work(c["rows"], c["Cin"], c["Cout"], outs, c["g"], c["bits"], e, c["residual"])
    else:   # what passes from one operator to the next need not pass through memory
        C, F, r = c["Cin"], c["width"], c["rows"]
        b1, f1 = _linear_work(r, C, 2 * F, 0, c["g"], c["bits"], 0, False)
        b2, f2 = _linear_work(r, F, C, C, c["g"], c["bits"], 0, False)
        b, f = b1 + b2 + 3 * e * r * C + e * r * C, f1 + f2
    return {"bytes": float(b), "flops": float(f)}


# ---- inputs ----

def _activations(gen, rows, C, dtype):
    """Hidden states: normal, one channel in a hundred 20 times as loud, every 64th row all zero
    (padding), rows of a few different sizes."""
    x = torch.randn((rows, C), generator=gen, device="cuda")
    gain = torch.ones(C, device="cuda")
    gain[torch.randperm(C, generator=gen, device="cuda")[:max(1, C // 100)]] = 20.0
    size = torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device="cuda"))
    size[63::64] = 0.0
    return (x * gain * size).to(TYPES[dtype])


def _weights(gen, Cin, Cout, g, bits):
    """A layer's weights: fp32 as loaded, and the codes and scales that a program keeps of them."""
    w = torch.randn((Cout, Cin), generator=gen, device="cuda") * 0.02
    bias = torch.randn((Cout,), generator=gen, device="cuda") * 0.1
    codes, scales = _quantize(w, g, 127 if bits == 8 else 7)
    return w, bias, codes, scales


def _plan(rows, Cin, Cout, g, bits, w, bias):
    from paper_2412_19867_amd import wq
    plan = wq.LinearPlan(rows, Cin, Cout, g, weight_bits=bits)
    blob = plan.alloc_blob()
    plan.weight_prepare(w, bias, blob)
    return plan, blob, plan.alloc_workspace()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": c, "x": _activations(gen, c["rows"], c["Cin"], c["dtype"])}
    if c["kind"] == "block" or c.get("residual"):
        outs = c["Cin"] if c["kind"] != "linear" else c["Cout"] // 2 if c["gated"] else c["Cout"]
        s["res"] = torch.randn((c["rows"], outs), generator=gen, device="cuda").to(TYPES[c["dtype"]])
    if c["kind"] in ("norm", "block"):
        s["gamma"] = 1.0 + 0.2 * torch.randn((c["Cin"],), generator=gen, device="cuda")
    sizes = {"linear": ((c["Cin"], c.get("Cout")),), "block": ((c["Cin"], 2 * c.get("width", 0)), (c.get("width"), c["Cin"]))}
    layers = []
    for Cin, Cout in sizes.get(c["kind"], ()):
        w, bias, codes, scales = _weights(gen, Cin, Cout, c["g"], c["bits"])
        # a program keeps its weights in the form that its calls read: codes and scales, or the library's blob
        layers.append(_plan(c["rows"], Cin, Cout, c["g"], c["bits"], w, bias) if own else (codes, scales, bias))
    s["layers"] = layers
    if own:
        if c["kind"] in ("norm", "quantize"):
            from paper_2412_19867_amd import wq
            plan = wq.LinearPlan(c["rows"], c["Cin"], 32, c["g"])
            s["plan"], s["ws"] = plan, plan.alloc_workspace()
        if c["kind"] in ("norm", "block"):
            s["h"] = torch.empty_like(s["x"])
        if c["kind"] == "block":
            s["mid"] = s["x"].new_empty((c["rows"], c["width"]))
            s["y"] = torch.empty_like(s["x"])
        if c["kind"] == "linear":
            s["y"] = s["x"].new_empty((c["rows"], c["Cout"] // 2 if c["gated"] else c["Cout"]))
    return s


# ---- plain forms ----

def _quantize(v, g, top=127):
    """Codes (int8, v's shape) and scales [rows][groups] of fp32 rows: the division in 64 bits and
    rounded to 32 is the correctly rounded one in 32."""
    v = v.reshape(v.shape[0], -1, g)
    a = v.abs().amax(dim=2)
    live = a >= top * TINY
    wide, tops = a.double(), torch.full_like(a, float(top), dtype=torch.float64)
    scale = torch.where(live, (wide / tops).float(), 0.0)
    r = torch.where(live, (tops / wide).float(), 0.0)
    return torch.round(v * r[..., None]).to(torch.int8).reshape(v.shape[0], -1), scale


def _values(codes, scales):
    """fp32 values that codes [rows][C] with scales [rows][groups] stand for."""
    rows, groups = scales.shape
    return (codes.float().view(rows, groups, -1) * scales[..., None]).view(rows, -1)


def _act(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0.0)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _plain_norm(x, res, gamma, g):
    h = x.float() if res is None else x.float() + res.float()
    wide = h.double()
    rho = (1.0 / torch.sqrt((wide * wide).mean(dim=1, keepdim=True) + EPS)).float()
    return (h.to(x.dtype), *_quantize(h * rho * gamma, g))


def _plain_product(codes, scales, layer, act, gated, res, dtype):
    wcodes, wscales, bias = layer
    z = torch.matmul(_values(codes, scales), _values(wcodes, wscales).t()) + bias
    if gated:
        gate, up = z.chunk(2, dim=1)
        z = _act(gate, act) * up
    else:
        z = _act(z, act)
    if res is not None:
        z = z + res.float()
    return z.to(dtype)


def _layout(plan, ws, rows):
    """The codes and scales in a workspace, as [rows][Cin / kstep][4][kstep / 4] and [rows][groups] views."""
    L = plan.layout
    codes = ws[L.ws_xq_off:L.ws_xq_off + L.P * L.Cin].view(torch.int8)
    codes = codes.view(L.Cin // L.kstep, 4, L.P, L.kstep // 4).permute(2, 0, 1, 3)
    scales = ws[L.ws_sx_off:L.ws_sx_off + L.P * L.groups * 4].view(torch.float32).view(L.groups, L.P).t()
    return codes[:rows], scales[:rows]


def _laid_out(codes, g):
    k = 32 if g == 32 else 64
    return codes.view(codes.shape[0], -1, 4, k // 4)


def run(state):
    s, c = state, state["case"]
    x, res, g = s["x"], s.get("res"), c["g"]
    if c["kind"] == "norm":
        if own:
            s["plan"].rms_norm_quantize(x, s["ws"], residual=res, gamma=s["gamma"], eps=EPS, out=s["h"])
            codes, scales = _layout(s["plan"], s["ws"], c["rows"])
            return {"h": s["h"], "codes": codes, "scales": scales}
        h, codes, scales = _plain_norm(x, res, s["gamma"], g)
        return {"h": h, "codes": _laid_out(codes, g), "scales": scales}
    if c["kind"] == "quantize":
        if own:
            s["plan"].quantize_rows(x, s["ws"])
            codes, scales = _layout(s["plan"], s["ws"], c["rows"])
            return {"codes": codes, "scales": scales}
        codes, scales = _quantize(x.float(), g)
        return {"codes": _laid_out(codes, g), "scales": scales}
    if c["kind"] == "linear":
        if own:
            plan, blob, ws = s["layers"][0]
            plan.linear(x, blob, ws, s["y"], activation=c["act"], gated=c["gated"], residual=res)
            return s["y"]
        return _plain_product(*_quantize(x.float(), g), s["layers"][0], c["act"], c["gated"], res, x.dtype)
    if own:
        (up, up_blob, up_ws), (down, down_blob, down_ws) = s["layers"]
        up.rms_norm_quantize(x, up_ws, residual=res, gamma=s["gamma"], eps=EPS, out=s["h"])
        up.matmul(up_ws, up_blob, s["mid"], activation="silu", gated=True)
        down.linear(s["mid"], down_blob, down_ws, s["y"], residual=s["h"])
        return {"h": s["h"], "y": s["y"]}
    h, codes, scales = _plain_norm(x, res, s["gamma"], g)
    mid = _plain_product(codes, scales, s["layers"][0], "silu", True, None, x.dtype)
    y = _plain_product(*_quantize(mid.float(), g), s["layers"][1], "none", False, h, x.dtype)
    return {"h": h, "y": y}


# ---- 64 bits ----

def _exact_codes(v, g):
    """(whole codes, scales), both fp64, of fp64 rows whose entries are fp32 numbers: the quantizer's
    definition, its roundings to fp32 taken literally."""
    fl = lambda t: t.to(torch.float32).to(torch.float64)   # noqa: E731
    blocks = torch.stack(torch.split(v, g, dim=1), dim=1)   # [rows][groups][g]
    top = torch.maximum(blocks.max(dim=2).values, -blocks.min(dim=2).values)
    seven = torch.full_like(top, 127.0)
    dead = top < 127.0 * TINY
    s, r = fl(torch.div(top, seven)).masked_fill(dead, 0.0), fl(torch.div(seven, top)).masked_fill(dead, 0.0)
    return torch.round(fl(blocks * r.unsqueeze(2))), s


def _exact_act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * (1.0 + torch.erf(z / math.sqrt(2.0))) / 2.0
    u = math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)
    return z * torch.sigmoid(2.0 * u)


def _exact_product(codes, scales, layer, act, gated, res):
    """codes [rows][groups][g] fp64; the sums of a group are whole numbers."""
    wcodes, wscales, bias = layer
    rows, groups, g = codes.shape
    z = bias.double().repeat(rows, 1)
    span = max(1, 2048 // g)   # a few groups at a time: their scaled codes side by side
    for k in range(0, groups, span):
        a = (codes[:, k:k + span] * scales[:, k:k + span, None]).reshape(rows, -1)
        b = wcodes[:, k * g:(k + span) * g].double().view(wcodes.shape[0], -1, g) * wscales[:, k:k + span, None].double()
        z += a @ b.reshape(wcodes.shape[0], -1).t()
    F = z.shape[1] // 2
    z = _exact_act(z[:, :F], act) * z[:, F:] if gated else _exact_act(z, act)
    return z if res is None else z + res.double()


def exact(case, seed):
    global own
    c, g = case, case["g"]
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    x = s["x"].double()
    if c["kind"] in ("norm", "block"):
        h = x + s["res"].double() if "res" in s else x
        h32 = h.float().double()   # the definition's fl(x + residual)
        rho = torch.rsqrt(h32.pow(2).sum(dim=1) / h32.shape[1] + EPS).float().double()
        v = (h32 * rho[:, None]).float().double()
        codes, scales = _exact_codes((v * s["gamma"].double()).float().double(), g)
        if c["kind"] == "norm":
            return {"h": h, "codes": None, "scales": scales}
        mid = _exact_product(codes, scales, s["layers"][0], "silu", True, None)
        mid = mid.to(TYPES[c["dtype"]]).double()   # the layers exchange values of their type
        low = h.to(TYPES[c["dtype"]])
        return {"h": h, "y": _exact_product(*_exact_codes(mid, g), s["layers"][1], "none", False, low)}
    codes, scales = _exact_codes(x, g)
    if c["kind"] == "quantize":
        return {"codes": None, "scales": scales}
    if 2.0 * c["rows"] * c["Cin"] * c["Cout"] > 6e11:
        return None
    return _exact_product(codes, scales, s["layers"][0], c["act"], c["gated"], s.get("res"))

"""Host-side tests of the linear layer's surroundings: the oracle's formulas pinned against others, and every
refusal of the C entry points and of the binding (no kernel is launched)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import linear_block as lb

OK, INVALID, UNSUPPORTED, NOT_PREPARED, WORKSPACE = 0, 1, 2, 4, 5


# ---- the oracle ----

def test_norm_formula():
    rng = np.random.default_rng(0)
    x, r = rng.standard_normal((5, 96), np.float32), rng.standard_normal((5, 96), np.float32)
    gamma = rng.standard_normal(96).astype(np.float32)
    h, v = lb.rms_norm(x, r, gamma, 1e-6)
    assert np.array_equal(h, x + r)
    hd = torch.from_numpy(h).double()
    want = hd / torch.sqrt((hd ** 2).mean(1, keepdim=True) + 1e-6) * torch.from_numpy(gamma).double()
    # rho, h rho and the product with gamma are rounded once each: three half steps of fp32
    assert (np.abs(v - want.numpy()) <= 3.001 * 2.0 ** -24 * np.abs(want.numpy())).all()
    h0, v0 = lb.rms_norm(np.zeros((2, 32), np.float32), None, None, 1e-6)
    assert not h0.any() and not v0.any()
    big = np.full((1, 64), 1e30, np.float32)   # its squares are beyond fp32
    assert np.allclose(lb.rms_norm(big, None, None, 1e-6)[1], 1.0, rtol=2.0 ** -23)


@pytest.mark.parametrize("act,f", [("none", lambda z: z), ("relu", torch.relu), ("silu", torch.nn.functional.silu),
                                   ("gelu", torch.nn.functional.gelu),
                                   ("gelu_tanh", lambda z: torch.nn.functional.gelu(z, approximate="tanh"))])
def test_activation_formulas(act, f):
    z = torch.cat([torch.linspace(-30, 30, 2001, dtype=torch.float64), torch.tensor([-800.0, 800.0, 0.0], dtype=torch.float64)])
    assert np.allclose(lb.activation(z.numpy(), act), f(z).numpy(), rtol=1e-10, atol=1e-13)


def test_product_and_epilogue_formulas():
    rng = np.random.default_rng(1)
    R, C, O, g = 3, 128, 64, 32
    xq, wq = rng.integers(-127, 128, (R, C)).astype(np.int8), rng.integers(-7, 8, (O, C)).astype(np.int8)
    sx, sw = rng.random((R, C // g)).astype(np.float32), rng.random((C // g, O)).astype(np.float32)
    bias = rng.standard_normal(O).astype(np.float32)
    z, S = lb.product(xq, sx, wq, sw, bias, g)
    xd = xq.astype(np.float64) * np.repeat(sx, g, 1)
    wd = wq.astype(np.float64) * np.repeat(sw.T, g, 1)
    assert np.allclose(z, xd @ wd.T + bias, rtol=1e-12, atol=1e-9) and (S >= np.abs(z) * (1 - 1e-12)).all()
    res = rng.standard_normal((R, O // 2))
    assert np.array_equal(lb.epilogue(z, "relu", True, res), np.maximum(z[:, :32], 0) * z[:, 32:] + res)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("gated", [False, True])
def test_the_bound_covers_an_fp32_evaluation_and_no_mistake(act, gated):
    """An evaluation in fp32 on the CPU stays inside the bound; one with a scale taken from the next group, and one
    rounded to bf16 on the way, do not."""
    rng = np.random.default_rng(2)
    R, C, O, g = 17, 512, 64, 64
    xq, wq = rng.integers(-127, 128, (R, C)).astype(np.int8), rng.integers(-127, 128, (O, C)).astype(np.int8)
    sx, sw = (rng.random((R, C // g)) * 0.02).astype(np.float32), (rng.random((C // g, O)) * 1e-3).astype(np.float32)
    bias = rng.standard_normal(O).astype(np.float32)
    res = rng.standard_normal((R, O // 2 if gated else O)).astype(np.float32)
    z, S = lb.product(xq, sx, wq, sw, bias, g)
    want, bound = lb.epilogue(z, act, gated, res), lb.epilogue_bound(z, S, C // g, act, gated, res, 2.0 ** -24)
    f = {"none": lambda t: t, "relu": torch.relu, "silu": lambda t: t / (1 + torch.exp(-t)),
         "gelu": lambda t: 0.5 * t * torch.erfc(t * -0.70710678),
         "gelu_tanh": lambda t: t / (1 + torch.exp(-1.5957691 * (t + 0.044715 * t * t * t)))}[act]

    def evaluate(sw_used, low=False):
        m = torch.zeros(R, O)
        for k in range(C // g):
            P = torch.from_numpy(xq[:, k * g:(k + 1) * g].astype(np.float32)) @ torch.from_numpy(wq[:, k * g:(k + 1) * g].astype(np.float32)).T
            m = m + P * (torch.from_numpy(sx[:, k, None]) * torch.from_numpy(sw_used[None, k]))
        m = m + torch.from_numpy(bias)
        if low:
            m = m.bfloat16().float()
        y = f(m[:, :O // 2]) * m[:, O // 2:] if gated else f(m)
        return (y + torch.from_numpy(res)).numpy()

    assert (np.abs(evaluate(sw) - want) <= bound).all()
    assert not (np.abs(evaluate(np.roll(sw, 1, 0)) - want) <= bound).all()
    assert not (np.abs(evaluate(sw, low=True) - want) <= bound).all()


# ---- refusals of the C entry points ----

class Plans:
    def __init__(self, wq):
        self.lin = wq.LinearPlan(10, 128, 64, 32)
        self.odd = wq.LinearPlan(10, 128, 48, 32)
        self.conv = wq.DirectPlan(1, 4, 4, 64, 64, 32)


PTR = 1 << 20   # an aligned address that is never read: every call below ends on the host


@pytest.fixture(scope="module")
def plans(wq):
    return Plans(wq)


def norm_args(of, **kw):
    a = dict(plan=of._h, stream=None, rows=10, type=1, x=PTR, xs=128, res=PTR, rs=128, gamma=PTR, eps=1e-6, sum=PTR, hs=128,
             ws=PTR, bytes=of.layout.ws_bytes)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("change,status", [
    (dict(plan=None), INVALID), (dict(x=None), INVALID), (dict(ws=None), INVALID),
    (dict(rows=11), INVALID), (dict(rows=-1), INVALID), (dict(type=3), INVALID), (dict(type=-1), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=-1e-6), INVALID), (dict(eps=1e-39), INVALID),
    (dict(eps=math.inf), INVALID), (dict(eps=math.nan), INVALID),
    (dict(xs=127), INVALID), (dict(rs=127), INVALID), (dict(hs=0), INVALID), (dict(xs=-128), INVALID),
    (dict(xs=1 << 62), INVALID), (dict(x=PTR + 1), INVALID), (dict(res=PTR + 1), INVALID), (dict(sum=PTR + 1), INVALID),
    (dict(type=0, x=PTR + 2), INVALID), (dict(gamma=PTR + 2), INVALID),
    (dict(bytes=100), WORKSPACE),
    (dict(rows=0), OK), (dict(rows=0, x=None, res=None, sum=None), OK), (dict(rows=0, bytes=100), WORKSPACE),
])
def test_norm_refusals(wq, plans, change, status):
    assert wq.lib().wq_rms_norm_quantize(*norm_args(plans.lin, **change)) == status


def quantize_args(of, **kw):
    a = dict(plan=of._h, stream=None, rows=10, type=1, x=PTR, xs=128, ws=PTR, bytes=of.layout.ws_bytes)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("change,status", [
    (dict(plan=None), INVALID), (dict(x=None), INVALID), (dict(ws=None), INVALID), (dict(rows=11), INVALID),
    (dict(type=7), INVALID), (dict(xs=100), INVALID), (dict(x=PTR + 1), INVALID), (dict(bytes=0), WORKSPACE),
    (dict(rows=0, x=None), OK),
])
def test_quantize_refusals(wq, plans, change, status):
    assert wq.lib().wq_linear_quantize(*quantize_args(plans.lin, **change)) == status


def matmul_args(of, **kw):
    L = of.layout
    a = dict(plan=of._h, stream=None, rows=10, ws=PTR, ws_bytes=L.ws_bytes, blob=PTR, blob_bytes=L.blob_bytes, act=2, gated=0,
             type=1, res=PTR, rs=L.Cout, y=PTR, ys=L.Cout)
    a.update(kw)
    return list(a.values())


MATMUL_REFUSALS = [
    (dict(plan=None), INVALID), (dict(ws=None), INVALID), (dict(blob=None), INVALID), (dict(y=None), INVALID),
    (dict(rows=11), INVALID), (dict(rows=-1), INVALID), (dict(act=5), INVALID), (dict(act=-1), INVALID), (dict(gated=2), INVALID),
    (dict(type=3), INVALID), (dict(ys=63), INVALID), (dict(rs=63), INVALID), (dict(gated=1, ys=31), INVALID),
    (dict(y=PTR + 1), INVALID), (dict(res=PTR + 1), INVALID), (dict(type=0, y=PTR + 2), INVALID),
    (dict(ws_bytes=1), WORKSPACE), (dict(blob_bytes=1), WORKSPACE),
    (dict(), NOT_PREPARED), (dict(gated=1, ys=32, rs=32), NOT_PREPARED), (dict(rows=1, ys=0, rs=0), NOT_PREPARED),
]


@pytest.mark.parametrize("change,status", MATMUL_REFUSALS)
def test_matmul_refusals(wq, plans, change, status):
    assert wq.lib().wq_linear_matmul(*matmul_args(plans.lin, **change)) == status


@pytest.mark.parametrize("change,status", MATMUL_REFUSALS)
def test_forward_refusals_of_the_product(wq, plans, change, status):
    a = dict(zip(("plan", "stream", "rows", "ws", "ws_bytes", "blob", "blob_bytes", "act", "gated", "type", "res", "rs", "y", "ys"),
                 matmul_args(plans.lin, **change)))
    assert wq.lib().wq_linear_forward(a["plan"], None, a["rows"], a["type"], PTR, 128, a["blob"], a["blob_bytes"], a["ws"],
                                      a["ws_bytes"], a["act"], a["gated"], a["res"], a["rs"], a["y"], a["ys"]) == status


def test_other_plans_are_refused(wq, plans):
    L = wq.lib()
    assert L.wq_rms_norm_quantize(*norm_args(plans.conv)) == UNSUPPORTED
    assert L.wq_linear_quantize(*quantize_args(plans.conv)) == UNSUPPORTED
    assert L.wq_linear_matmul(*matmul_args(plans.conv)) == UNSUPPORTED
    assert L.wq_linear_matmul(*matmul_args(plans.odd, gated=1, ys=24, rs=24)) == UNSUPPORTED   # 48 channels: no two halves of whole blocks
    assert L.wq_linear_matmul(*matmul_args(plans.odd)) == NOT_PREPARED


# ---- the binding's ----

def test_binding_refuses_what_is_not_a_device_tensor(wq, plans):
    x, ws = torch.zeros(4, 128), torch.zeros(1 << 16, dtype=torch.uint8)
    for call in (lambda: plans.lin.rms_norm_quantize(x, ws), lambda: plans.lin.quantize_rows(x, ws),
                 lambda: plans.lin.matmul(ws, ws, x), lambda: plans.lin.linear(x, ws, ws, x),
                 lambda: plans.lin.quantize_rows("x", None)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError, match="activation"):
        plans.lin.matmul(ws, ws, x, activation="swish")
    with pytest.raises(wq.WqError):
        wq.LinearPlan(4, 100, 32, 32)
    with pytest.raises(wq.WqError):
        wq.LinearPlan(4, 128, 32, 32, weight_bits=3)

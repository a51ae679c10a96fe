"""Host-side tests of the linear layer in 8-bit floating point and of the layer norm: the oracle's formulas pinned against others,
and every refusal of the C entry points and of the binding (no kernel is launched)."""
import math

import numpy as np
import pytest
import torch

from oracle import fp8_block as fb

OK, INVALID, UNSUPPORTED, NOT_PREPARED, WORKSPACE = 0, 1, 2, 4, 5
PTR = 1 << 20   # an aligned address that is never read: every call below ends on the host


# ---- the oracle ----

def test_codes_are_the_nearest_numbers():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(20000) * s for s in (1e-3, 1.0, 100.0)] + [np.arange(-3680, 3681) / 8.0, np.arange(-600, 600) / 4096.0])
    x = np.clip(x, -463.9, 463.9).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn)
    assert np.array_equal(fb.encode(x), want.view(torch.uint8).numpy())
    assert np.array_equal(fb.decode(fb.encode(x)), want.double().numpy())
    assert fb.encode([464.0, 464.1, np.nan, np.inf, -np.inf, 448.0, -0.0]).tolist() == [126, 127, 127, 127, 255, 126, 128]


def test_scales_are_the_smallest_powers_of_two():
    tops = np.array([0.0, 1e-38, 448.0, np.nextafter(np.float32(448), np.float32(500)), 1.0, 1.75, 1.7500001, 3.4e38, np.inf])
    s = fb.pow2_scale(tops)
    assert np.array_equal(s, 2.0 ** np.array([-126, -126, 0, 1, -8, -8, -7, 120, 120]))
    assert (tops[:8] <= 448 * s[:8]).all()


@pytest.mark.parametrize("act,f", [("none", lambda z: z), ("relu", torch.relu), ("silu", torch.nn.functional.silu),
                                   ("gelu", torch.nn.functional.gelu),
                                   ("gelu_tanh", lambda z: torch.nn.functional.gelu(z, approximate="tanh"))])
def test_slopes_are_the_derivatives(act, f):
    z = torch.cat([torch.linspace(-12, 12, 601, dtype=torch.float64), torch.tensor([0.0, -300.0, 300.0], dtype=torch.float64)]).requires_grad_()
    f(z).sum().backward()
    assert np.allclose(fb.slope(z.detach().numpy(), act), z.grad.numpy(), rtol=1e-9, atol=1e-12)
    # and the gate's two halves, against differences
    rng = np.random.default_rng(1)
    pre, dy, d = rng.standard_normal((3, 8)) + 0.3, rng.standard_normal((3, 4)), rng.standard_normal((3, 8))
    y = lambda p: fb.epilogue(p, act, True, None)   # noqa: E731
    want = (dy * (y(pre + 1e-6 * d) - y(pre - 1e-6 * d)) / 2e-6).sum()
    assert abs((fb.gate_grad(dy, pre, act, True) * d).sum() - want) < 1e-6 * (1 + abs(want))


def test_layer_norm_and_its_gradient():
    rng = np.random.default_rng(2)
    x, res, dy = (rng.standard_normal((5, 37)).astype(np.float32) for _ in range(3))
    gamma, beta = (rng.standard_normal(37).astype(np.float32) for _ in range(2))
    h, v = fb.layer_norm(x, res, gamma, beta, 1e-3)
    t = torch.from_numpy(h).double().requires_grad_()
    g, b = torch.from_numpy(gamma).double().requires_grad_(), torch.from_numpy(beta).double().requires_grad_()
    y = torch.nn.functional.layer_norm(t, (37,), g, b, 1e-3)
    # off, r, off r, times gamma, plus beta: a half step of fp32 each, relative to the product and the sum
    assert (np.abs(v - y.detach().numpy()) <= 6 * 2.0 ** -24 * (np.abs(y.detach().numpy()) + np.abs(beta))).all()
    y.backward(torch.from_numpy(dy).double())
    dx, dgamma, dbeta = fb.layer_norm_grad(dy, h, gamma, None, 1e-3)
    for got, want in ((dx, t.grad), (dgamma, g.grad), (dbeta, b.grad)):
        assert np.allclose(got, want.numpy(), rtol=1e-9, atol=1e-12)
    # a row far from zero, and a constant one
    far = np.stack([1e6 + rng.standard_normal(64), np.full(64, 3e7)]).astype(np.float32)
    assert not fb.layer_norm(far, None, None, None, 1e-5)[1][1].any()


def test_blocks_and_products():
    rng = np.random.default_rng(3)
    w, x = rng.standard_normal((200, 150)), rng.standard_normal((3, 150))
    codes, s = fb.quantize_blocks(w)
    assert s.shape == (2, 2)
    assert (np.abs(fb.block_values(codes, s) - w) <= 2.0 ** -4 * np.abs(w) + 2.0 ** -10 * s.max()).all()
    z, S = fb.product(fb.through(x), fb.block_values(codes, s), None)
    assert np.allclose(z, x @ w.T, atol=0.2 * np.sqrt(150)) and (S >= np.abs(z)).all()


# ---- refusals of the C entry points ----

class Plans:
    def __init__(self, wq):
        self.p = wq.Fp8LinearPlan(10, 200, 192, backward=True)
        self.fwd = wq.Fp8LinearPlan(10, 200, 192)
        self.any = wq.Fp8LinearPlan(10, 200, 96, backward=True, fp32_scales=True)


@pytest.fixture(scope="module")
def plans(wq):
    return Plans(wq)


def call(f, order, defaults, **change):
    a = dict(defaults)
    assert not set(change) - set(a)
    a.update(change)
    return f(*[a[k] for k in order.split()])


@pytest.mark.parametrize("args,status", [
    ((0, 8, 8, 0, 0), INVALID), ((8, 0, 8, 0, 0), INVALID), ((8, 8, 0, 0, 0), INVALID), ((8, 8, 8, 2, 0), INVALID), ((8, 8, 8, 0, 2), INVALID),
    ((-1, 8, 8, 0, 0), INVALID), ((1, 1, 1, 1, 1), OK), ((1 << 24, 128, 8, 0, 0), UNSUPPORTED), ((1, 1 << 20, 1 << 12, 0, 0), UNSUPPORTED),
    ((1 << 20, 128, 4096, 1, 0), UNSUPPORTED), ((1 << 20, 128, 4096, 0, 0), OK), ((1, 1 << 15, 1 << 15, 1, 0), OK),
])
def test_plan_refusals(wq, args, status):
    import ctypes
    h = ctypes.c_void_p()
    assert wq.lib().wq_fp8_plan_create(ctypes.byref(h), *args) == status
    assert bool(h) == (status == OK)
    if h:
        assert wq.lib().wq_fp8_plan_destroy(h) == OK
    assert wq.lib().wq_fp8_plan_create(None, 1, 1, 1, 0, 0) == INVALID
    assert wq.lib().wq_fp8_plan_layout(None, None) == INVALID and wq.lib().wq_fp8_plan_destroy(None) == INVALID


PREPARE = "plan stream type w ws bias blob bytes"


@pytest.mark.parametrize("change,status", [
    (dict(plan=None), INVALID), (dict(w=None), INVALID), (dict(blob=None), INVALID), (dict(blob=PTR + 8), INVALID), (dict(type=3), INVALID),
    (dict(ws=199), INVALID), (dict(w=PTR + 2), INVALID), (dict(bias=PTR + 2), INVALID), (dict(bytes=100), WORKSPACE)])
def test_weight_prepare_refusals(wq, plans, change, status):
    d = dict(plan=plans.p._h, stream=None, type=0, w=PTR, ws=200, bias=PTR, blob=PTR, bytes=plans.p.layout.blob_bytes)
    assert call(wq.lib().wq_fp8_weight_prepare, PREPARE, d, **change) == status


LOAD = "plan stream codes cs kind scales bias blob bytes"


@pytest.mark.parametrize("change,status", [
    (dict(plan=None), INVALID), (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(blob=None), INVALID), (dict(kind=2), INVALID),
    (dict(cs=199), INVALID), (dict(scales=PTR + 2), INVALID), (dict(bytes=0), WORKSPACE), (dict(bias=PTR + 1), INVALID)])
def test_weight_load_refusals(wq, plans, change, status):
    d = dict(plan=plans.any._h, stream=None, codes=PTR, cs=200, kind=0, scales=PTR, bias=PTR, blob=PTR, bytes=plans.any.layout.blob_bytes)
    assert call(wq.lib().wq_fp8_weight_load, LOAD, d, **change) == status
    if not change.keys() & {"plan"}:   # a plan whose scales are powers of two takes no others
        d.update(plan=plans.p._h, bytes=plans.p.layout.blob_bytes)
        assert call(wq.lib().wq_fp8_weight_load, LOAD, d) == UNSUPPORTED


QUANT = "plan stream rows type x xs ws bytes"


@pytest.mark.parametrize("change,status", [
    (dict(plan=None), INVALID), (dict(x=None), INVALID), (dict(ws=None), INVALID), (dict(ws=PTR + 8), INVALID), (dict(rows=11), INVALID),
    (dict(rows=-1), INVALID), (dict(type=3), INVALID), (dict(xs=199), INVALID), (dict(x=PTR + 1), INVALID), (dict(bytes=1), WORKSPACE),
    (dict(rows=0, x=None), OK), (dict(xs=1 << 60), INVALID)])
def test_quantize_refusals(wq, plans, change, status):
    d = dict(plan=plans.fwd._h, stream=None, rows=10, type=1, x=PTR, xs=200, ws=PTR, bytes=plans.fwd.layout.ws_bytes)
    assert call(wq.lib().wq_fp8_quantize, QUANT, d, **change) == status


NORMQ = "plan stream rows type x xs res rs gamma beta eps sum ss ws bytes"


@pytest.mark.parametrize("change,status", [
    (dict(plan=None), INVALID), (dict(x=None), INVALID), (dict(ws=None), INVALID), (dict(rows=11), INVALID), (dict(rows=-1), INVALID),
    (dict(type=5), INVALID), (dict(xs=1), INVALID), (dict(rs=1), INVALID), (dict(ss=1), INVALID), (dict(gamma=PTR + 1), INVALID),
    (dict(beta=PTR + 2), INVALID), (dict(eps=0.0), INVALID), (dict(eps=math.nan), INVALID), (dict(eps=math.inf), INVALID), (dict(eps=-1.0), INVALID),
    (dict(bytes=0), WORKSPACE), (dict(rows=0, x=None, res=None, sum=None), OK), (dict(res=PTR + 1), INVALID)])
def test_layer_norm_quantize_refusals(wq, plans, change, status):
    d = dict(plan=plans.fwd._h, stream=None, rows=10, type=1, x=PTR, xs=200, res=PTR, rs=200, gamma=PTR, beta=PTR, eps=1e-5, sum=PTR, ss=200,
             ws=PTR, bytes=plans.fwd.layout.ws_bytes)
    assert call(wq.lib().wq_fp8_layer_norm_quantize, NORMQ, d, **change) == status


MATMUL = "plan stream rows ws ws_bytes blob blob_bytes act gated type res rs pre ps y ys"
FORWARD = "plan stream rows type x xs blob blob_bytes ws ws_bytes act gated res rs pre ps y ys"


@pytest.mark.parametrize("change,status", [
    (dict(plan=None), INVALID), (dict(ws=None), INVALID), (dict(blob=None), INVALID), (dict(y=None), INVALID), (dict(rows=11), INVALID),
    (dict(rows=-1), INVALID), (dict(act=5), INVALID), (dict(act=-1), INVALID), (dict(gated=2), INVALID), (dict(type=3), INVALID),
    (dict(ys=191), INVALID), (dict(rs=191), INVALID), (dict(ps=191), INVALID), (dict(gated=1, ys=95), INVALID), (dict(y=PTR + 1), INVALID),
    (dict(pre=PTR + 1), INVALID), (dict(type=0, y=PTR + 2), INVALID), (dict(ws_bytes=1), WORKSPACE), (dict(blob_bytes=1), WORKSPACE),
    (dict(), NOT_PREPARED), (dict(gated=1, ys=96, rs=96), NOT_PREPARED), (dict(rows=1, ys=0, rs=0, ps=0), NOT_PREPARED),
    (dict(blob=PTR + 8), INVALID), (dict(ws=PTR + 4), INVALID)])
def test_product_refusals(wq, plans, change, status):
    L = plans.fwd.layout
    d = dict(plan=plans.fwd._h, stream=None, rows=10, type=1, x=PTR, xs=200, blob=PTR, blob_bytes=L.blob_bytes, ws=PTR, ws_bytes=L.ws_bytes,
             act=2, gated=0, res=PTR, rs=192, pre=PTR, ps=192, y=PTR, ys=192)
    assert call(wq.lib().wq_fp8_matmul, MATMUL, d, **change) == status
    assert call(wq.lib().wq_fp8_forward, FORWARD, d, **change) == status


def test_a_gate_needs_whole_halves(wq, plans):
    L = plans.any.layout   # 96 columns: halves of 48
    d = dict(plan=plans.any._h, stream=None, rows=10, type=1, x=PTR, xs=200, blob=PTR, blob_bytes=L.blob_bytes, ws=PTR, ws_bytes=L.ws_bytes,
             act=2, gated=1, res=None, rs=0, pre=None, ps=0, y=PTR, ys=48)
    assert call(wq.lib().wq_fp8_matmul, MATMUL, d) == UNSUPPORTED
    assert call(wq.lib().wq_fp8_forward, FORWARD, d) == UNSUPPORTED


BACK = "plan stream rows type x xs dy dys pre ps blob blob_bytes ws ws_bytes act gated dx dxs wt dw dws db acc"


@pytest.mark.parametrize("change,status", [
    (dict(plan=None), INVALID), (dict(rows=11), INVALID), (dict(rows=-1), INVALID), (dict(type=4), INVALID), (dict(act=9), INVALID),
    (dict(gated=3), INVALID), (dict(ws=None), INVALID), (dict(ws=PTR + 8), INVALID), (dict(acc=2), INVALID), (dict(db=PTR + 2), INVALID),
    (dict(wt=2), INVALID), (dict(dws=199), INVALID), (dict(wt=0, dw=PTR + 2), INVALID), (dict(blob=None), INVALID), (dict(dxs=199), INVALID),
    (dict(dx=PTR + 1), INVALID), (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(pre=None), INVALID), (dict(dys=191), INVALID),
    (dict(xs=199), INVALID), (dict(ps=191), INVALID), (dict(gated=1, dys=95), INVALID), (dict(ws_bytes=3), WORKSPACE), (dict(blob_bytes=3), WORKSPACE),
    (dict(), NOT_PREPARED), (dict(gated=1, dys=96), NOT_PREPARED), (dict(act=0, pre=None), NOT_PREPARED), (dict(dw=None, x=None), NOT_PREPARED),
    (dict(dx=None, dw=None, db=None), OK), (dict(dx=None, blob=None, rows=0, acc=1), OK), (dict(dx=None, dw=None, db=None, rows=0, dy=None, pre=None), OK)])
def test_backward_refusals(wq, plans, change, status):
    L = plans.p.layout
    d = dict(plan=plans.p._h, stream=None, rows=10, type=1, x=PTR, xs=200, dy=PTR, dys=192, pre=PTR, ps=192, blob=PTR, blob_bytes=L.blob_bytes,
             ws=PTR, ws_bytes=L.ws_bytes, act=2, gated=0, dx=PTR, dxs=200, wt=1, dw=PTR, dws=200, db=PTR, acc=0)
    assert call(wq.lib().wq_fp8_backward, BACK, d, **change) == status
    if not change:   # a plan without room for gradients
        d.update(plan=plans.fwd._h)
        assert call(wq.lib().wq_fp8_backward, BACK, d) == UNSUPPORTED


NORM = "stream rows C type x xs res rs gamma beta eps sum ss y ys"


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), INVALID), (dict(C=0), INVALID), (dict(type=3), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(xs=63), INVALID),
    (dict(rs=63), INVALID), (dict(ss=63), INVALID), (dict(ys=63), INVALID), (dict(x=PTR + 1), INVALID), (dict(y=PTR + 1), INVALID),
    (dict(gamma=PTR + 2), INVALID), (dict(beta=PTR + 2), INVALID), (dict(eps=0.0), INVALID), (dict(eps=math.inf), INVALID),
    (dict(sum=PTR), INVALID), (dict(rows=0, x=None, y=None), OK), (dict(rows=1 << 26), UNSUPPORTED),
    (dict(rows=1 << 24, C=4096, xs=4096, rs=4096, ss=4096, ys=4096), UNSUPPORTED)])
def test_layer_norm_refusals(wq, change, status):
    d = dict(stream=None, rows=4, C=64, type=1, x=PTR, xs=64, res=PTR, rs=64, gamma=PTR, beta=PTR, eps=1e-5, sum=PTR + 4096, ss=64, y=PTR, ys=64)
    assert call(wq.lib().wq_layer_norm, NORM, d, **change) == status


NGRAD = "stream rows C type dy dys h hs gamma eps res rs dx dxs dgamma dbeta acc ws bytes"


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), INVALID), (dict(C=0), INVALID), (dict(type=-1), INVALID), (dict(dy=None), INVALID), (dict(h=None), INVALID), (dict(ws=None), INVALID),
    (dict(ws=PTR + 8), INVALID), (dict(acc=2), INVALID), (dict(eps=0.0), INVALID), (dict(dys=1), INVALID), (dict(hs=1), INVALID), (dict(rs=1), INVALID),
    (dict(dxs=1), INVALID), (dict(dgamma=PTR + 1), INVALID), (dict(dbeta=PTR + 1), INVALID), (dict(gamma=PTR + 1), INVALID), (dict(bytes=0), WORKSPACE),
    (dict(dx=None, dgamma=None, dbeta=None), OK), (dict(rows=0, dy=None, h=None, acc=1), OK)])
def test_layer_norm_grad_refusals(wq, change, status):
    d = dict(stream=None, rows=4, C=64, type=1, dy=PTR, dys=64, h=PTR, hs=64, gamma=PTR, eps=1e-5, res=PTR, rs=64, dx=PTR, dxs=64, dgamma=PTR,
             dbeta=PTR, acc=0, ws=PTR, bytes=1 << 20)
    assert call(wq.lib().wq_layer_norm_grad, NGRAD, d, **change) == status


def test_layer_norm_workspace(wq):
    import ctypes
    size, f = ctypes.c_uint64(), wq.lib().wq_layer_norm_workspace
    assert f(-1, 8, ctypes.byref(size)) == INVALID and f(1, 0, ctypes.byref(size)) == INVALID and f(1, 8, None) == INVALID
    assert f(1 << 22, 9000, ctypes.byref(size)) == UNSUPPORTED and f(1 << 21, 9000, ctypes.byref(size)) == OK
    assert f(1 << 26, 8, ctypes.byref(size)) == UNSUPPORTED and f(8, (1 << 30) + 1, ctypes.byref(size)) == UNSUPPORTED
    for C in (1, 512, 8192, 16384, 20000):   # more rows need as much or more
        last = 0
        for rows in (0, 1, 3, 4, 100, 1000, 5000, 100000):
            assert f(rows, C, ctypes.byref(size)) == OK and size.value >= last
            last = size.value


# ---- the binding's ----

def test_binding_refuses_what_is_not_a_device_tensor(wq, plans):
    x, ws = torch.zeros(4, 200), torch.zeros(1 << 16, dtype=torch.uint8)
    norm = wq.LayerNormPlan(4, 200)
    for f in (lambda: plans.p.quantize_rows(x, ws), lambda: plans.p.layer_norm_quantize(x, ws), lambda: plans.p.matmul(ws, ws, x),
              lambda: plans.p.linear(x, ws, ws, x), lambda: plans.p.backward(x, x, ws, ws), lambda: plans.p.weight_prepare(x, None, ws),
              lambda: plans.p.weight_load(x, x, None, ws), lambda: norm.forward(x, x), lambda: norm.backward(x, x, ws),
              lambda: norm.forward("x", None)):
        with pytest.raises(TypeError):
            f()
    with pytest.raises(ValueError, match="activation"):
        plans.p.matmul(ws, ws, x, activation="swish")
    with pytest.raises(wq.WqError):
        wq.Fp8LinearPlan(4, 0, 8)
    with pytest.raises(wq.WqError):
        wq.LayerNormPlan(4, 0)

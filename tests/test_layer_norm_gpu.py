"""Layer norm on the GPU, into rows and into codes, and its gradient, against 64 bits (oracle.fp8_block)."""
import numpy as np
import pytest
import torch

from oracle import fp8_block as fb
from test_fp8_gpu import HALF, NAMES, U, between, bits, check, f64, hidden, rows_of

pytestmark = pytest.mark.gpu

# rows, rows of the plan, C
NORMS = [(1, 1, 1), (1, 3, 7), (1, 1, 4096), (3, 3, 513), (5, 8, 96), (7, 7, 640), (16, 16, 4096), (9, 33, 1281), (130, 130, 320), (2, 2, 8192),
         (17, 17, 5120), (3, 3, 16385), (2, 4, 33280), (1, 1, 70001), (65, 65, 2047), (777, 777, 130), (1300, 1300, 24),
         (5, 5, 8200), (4, 4, 12001), (3, 3, 16384), (3, 3, 24000), (2, 2, 32767)]   # over 16 waves, with two pieces a lane and with four


def vectors(rng, C):
    return (1.0 + 0.2 * rng.standard_normal(C)).astype(np.float32), (0.3 * rng.standard_normal(C)).astype(np.float32)


def on(v):
    return None if v is None else torch.from_numpy(v).cuda()


def near(x, res, gamma, beta, eps):
    """(h, v, how far fp32 rounding may move v): the statistics' 64 bits may fall on either side of a rounding to 32, so o and r may each
    be a step off, and the product, its product with gamma and the sum with beta a half step each."""
    h, v = fb.layer_norm(x, res, gamma, beta, eps)
    b = 0.0 if beta is None else np.abs(beta)
    return h, v, 8 * U * (np.abs(v) + b)


def check_codes(plan, ws, n, v, e):
    """Codes and scales of v, which may be off by e: equal wherever both ends have the same code, and between the ends' elsewhere."""
    got, s = plan.workspace_views(ws)
    lo, hi = fb.quantize_rows(np.abs(v) - e), fb.quantize_rows(np.abs(v) + e)
    assert ((f64(s[:n]) >= lo[1]) & (f64(s[:n]) <= hi[1])).all()
    C = v.shape[1]
    values = np.abs(fb.row_values(bits(got[:n]).reshape(n, -1), f64(s[:n]), C))
    ends = [np.abs(fb.row_values(*q, C)) for q in (lo, hi)]
    assert ((values >= np.minimum(*ends)) & (values <= np.maximum(*ends))).all()
    assert (bits(got[:n]).reshape(n, -1)[:, C:] == 0).all()   # the last group is filled up
    codes, scales = fb.quantize_rows(v)
    same = (bits(got[:n]).reshape(n, -1) & 127) == (codes & 127)
    assert same.mean() >= 0.999   # a last bit decides few of them


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("case", NORMS, ids=lambda c: "%dof%d_%d" % c)
def test_forward(wq, case, dtype):
    n, R, C = case
    print(case, dtype, flush=True)
    rng = np.random.default_rng(n * 131 + C)
    norm, plan = wq.LayerNormPlan(R, C), wq.Fp8LinearPlan(R, C, 8)
    x, res = hidden(rng, n, C, dtype), hidden(rng, n, C, dtype)
    gamma, beta = vectors(rng, C)
    for with_res, with_gamma, with_beta, strided, sum_into in ((1, 1, 1, 0, "out"), (0, 0, 0, 0, None), (1, 0, 1, 1, "residual"), (1, 1, 0, 2, "x"),
                                                               (0, 1, 1, 1, "out")):
        # 1: a row stride of whole 16-byte pieces, 2: odd strides and offsets
        stride, off = ((C, 0), (C + 16, 8), (C + 3, 1))[strided]
        g, b = gamma if with_gamma else None, beta if with_beta else None
        h, v, e = near(f64(x), f64(res) if with_res else None, g, b, 1e-5)
        for codes in (False, True):
            xd, rd = rows_of(x, stride, off), rows_of(res, stride, off) if with_res else None
            out = {"out": rows_of(torch.zeros_like(x), stride, off), "residual": rd, "x": xd, None: None}[sum_into]
            if codes:
                ws = plan.alloc_workspace()
                ws.fill_(0xA5)
                before = [bits(t[n:]).tobytes() for t in plan.workspace_views(ws)]
                plan.layer_norm_quantize(xd, ws, residual=rd, gamma=on(g), beta=on(b), eps=1e-5, out=out)
                torch.cuda.synchronize()
                check_codes(plan, ws, n, v, e)
                assert before == [bits(t[n:]).tobytes() for t in plan.workspace_views(ws)]   # rows behind the last one stay
            else:
                y = rows_of(torch.zeros_like(x), stride, off)
                if sum_into is None:
                    y = xd   # in place
                norm.forward(xd, y, gamma=on(g), beta=on(b), eps=1e-5, residual=rd, out=out)
                torch.cuda.synchronize()
                check(y, v.astype(np.float64), e)
                if stride > C:
                    assert bool(between(y, stride, off).isnan().all())
            if out is not None:
                assert torch.equal(out.cpu(), torch.from_numpy(h).to(x.dtype))
                if stride > C:
                    assert bool(between(out, stride, off).isnan().all())


def test_extreme_rows(wq):
    """Rows far from zero, constant ones, one value in a row of zeros, squares beyond fp32, and what is not a number."""
    C = 512
    rng = np.random.default_rng(1)
    x = np.zeros((8, C), np.float32)
    x[0] = 1e5 + rng.standard_normal(C)
    x[1] = 3e7
    x[2, 7] = 1.0
    x[3] = 1e30 * rng.standard_normal(C)
    x[4] = 1e-30 * rng.standard_normal(C)
    x[5, 0], x[5, 1:] = 1e6, rng.standard_normal(C - 1)   # the first element, from which the sums start, is the outlier
    x[6, 3] = np.nan
    x[7, 9] = np.inf
    norm = wq.LayerNormPlan(8, C)
    for eps in (1e-5, 2.0 ** -126, 1e30):
        y = torch.empty((8, C), device="cuda")
        norm.forward(torch.from_numpy(x).cuda(), y, eps=eps)
        h, v, e = near(x[:6], None, None, None, eps)
        check(y[:6], v.astype(np.float64), e)
        assert bool(y[6:].isnan().all())


def grad_bounds(dy, h, gamma, res, eps):
    dx, dgamma, dbeta = fb.layer_norm_grad(dy, h, gamma, res, eps)
    off = h - h.mean(1, keepdims=True)
    r = 1 / np.sqrt((off * off).mean(1, keepdims=True) + eps)
    n, g = off * r, dy if gamma is None else dy * gamma.astype(np.float64)
    mg, mgn = g.mean(1, keepdims=True), (g * n).mean(1, keepdims=True)
    # The means are sums in 64 bits of g = fl(dy gamma), each off by up to U |g|: they are off by up to U mean|g| and U mean|g n|, however
    # small the terms of either sign leave them.  They, n (two roundings), its product with the second mean and two differences are
    # rounded to fp32, as are r, the product with it and the last sum.
    means = U * (np.abs(g).mean(1, keepdims=True) + np.abs(n) * np.abs(g * n).mean(1, keepdims=True))
    ex = 10 * U * (r * (np.abs(g) + np.abs(mg) + np.abs(n * mgn)) + (0 if res is None else np.abs(res))) + r * means
    # a unit's rows one after the other in fp32, then 64 bits; n is off by two roundings
    rows = dy.shape[0]
    ew = (rows / 100 + 30) * U * np.abs(dy * n).sum(0)
    eb = (rows / 100 + 30) * U * np.abs(dy).sum(0)
    return (dx, ex), (dgamma, ew), (dbeta, eb)


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("case", NORMS + [(2100, 2100, 640), (600, 600, 4100)], ids=lambda c: "%dof%d_%d" % c)
def test_backward(wq, case, dtype):
    n, R, C = case
    print(case, dtype, flush=True)
    rng = np.random.default_rng(n * 7 + C)
    norm = wq.LayerNormPlan(R, C)
    dy, h, res = hidden(rng, n, C, dtype, 0.01), hidden(rng, n, C, dtype), hidden(rng, n, C, dtype, 0.01)
    gamma, _ = vectors(rng, C)
    for with_gamma, with_res, strided, into in ((1, 0, 0, None), (0, 1, 1, "dy"), (1, 1, 2, "h"), (1, 1, 0, "res")):
        stride, off = ((C, 0), (C + 16, 8), (C + 3, 1))[strided]
        g = gamma if with_gamma else None
        wants = grad_bounds(f64(dy), f64(h), g, f64(res) if with_res else None, 1e-5)
        dyd, hd, rd = rows_of(dy, stride, off), rows_of(h, stride, off), rows_of(res, stride, off) if with_res else None
        dx = {None: rows_of(torch.zeros_like(dy), stride, off), "dy": dyd, "h": hd, "res": rd}[into]
        dgamma, dbeta = torch.full((C,), float("nan"), device="cuda"), torch.full((C,), float("nan"), device="cuda")
        ws = norm.alloc_workspace()
        ws.fill_(0xFF)
        norm.backward(dyd, hd, ws, dx=dx, gamma=on(g), eps=1e-5, residual_grad=rd, dgamma=dgamma, dbeta=dbeta)
        torch.cuda.synchronize()
        for got, (want, e) in zip((dx, dgamma, dbeta), wants):
            check(got, want, e)
        if stride > C:
            assert bool(between(dx, stride, off).isnan().all())
        if into is None:   # the same bits again, one at a time, and added to what is there
            one = torch.empty_like(dgamma)
            norm.backward(dyd, hd, ws, gamma=on(g), eps=1e-5, dgamma=one)
            assert torch.equal(one, dgamma)
            norm.backward(dyd, hd, ws, gamma=on(g), eps=1e-5, dbeta=one)
            assert torch.equal(one, dbeta)
            only = torch.empty_like(dx)
            norm.backward(dyd, hd, ws, dx=only, gamma=on(g), eps=1e-5)
            assert torch.equal(only, dx)
            norm.backward(dyd, hd, ws, gamma=on(g), eps=1e-5, dgamma=dgamma, dbeta=dbeta, accumulate=True)
            check(dgamma, 2 * wants[1][0], 2 * wants[1][1])
            check(dbeta, 2 * wants[2][0], 2 * wants[2][1])


def test_gradient_against_differences(wq):
    rng = np.random.default_rng(4)
    n, C = 6, 200
    norm = wq.LayerNormPlan(n, C)
    x, dy, d = (rng.standard_normal((n, C)).astype(np.float32) for _ in range(3))
    gamma, beta = vectors(rng, C)
    dx = torch.empty((n, C), device="cuda")
    norm.backward(on(dy), on(x), norm.alloc_workspace(), dx=dx, gamma=on(gamma))
    loss = []
    step = 2.0 ** -7
    for sign in (1, -1):
        y = torch.empty((n, C), device="cuda")
        norm.forward(on((x + sign * step * d).astype(np.float32)), y, gamma=on(gamma), beta=on(beta))
        loss.append((f64(y) * dy).sum())
    got, want = (loss[0] - loss[1]) / (2 * step), (f64(dx) * d).sum()
    # y's rounding over the step, and the third derivative's share, about the step's square of the sum of the terms
    assert abs(got - want) <= 8 * U * np.abs(dy).sum() * 4 / step + 20 * step ** 2 * np.abs(dy * d).sum()


def test_no_rows(wq):
    norm = wq.LayerNormPlan(4, 33)
    e = torch.empty((0, 33), device="cuda", dtype=torch.bfloat16)
    norm.forward(e, torch.empty_like(e))
    ws = norm.alloc_workspace()
    a, b = torch.ones(33, device="cuda"), torch.ones(33, device="cuda")
    norm.backward(e, e, ws, dx=torch.empty_like(e), dgamma=a, dbeta=b, accumulate=True)
    assert bool((a == 1).all()) and bool((b == 1).all())
    norm.backward(e, e, ws, dx=torch.empty_like(e), dgamma=a, dbeta=b)
    assert not a.any() and not b.any()


def test_rows_far_apart_and_other_streams(wq):
    rng = np.random.default_rng(8)
    n, C, stride = 9, 200, 1 << 27
    norm = wq.LayerNormPlan(n, C)
    big = torch.empty((n * stride,), dtype=torch.bfloat16, device="cuda").view(n, stride)
    x = hidden(rng, n, C, "bf16")
    xd, yd, dxd = big[:, :C], big[:, 300:300 + C], big[:, 600:600 + C]
    xd.copy_(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    norm.forward(xd, yd, stream=s)
    s.synchronize()
    _, v, e = near(f64(x), None, None, None, 1e-5)
    check(yd, v.astype(np.float64), e)
    ws = norm.alloc_workspace()
    torch.cuda.synchronize()
    norm.backward(yd, xd, ws, dx=dxd, stream=s)
    s.synchronize()
    (dx, ex), _, _ = grad_bounds(f64(yd), f64(x), None, None, 1e-5)
    check(dxd, dx, ex)
    with pytest.raises(ValueError):
        norm.forward(xd, yd[:3])
    with pytest.raises(TypeError):
        norm.forward(xd, yd.float())
    with pytest.raises(TypeError):
        norm.backward(yd, None, ws, dx=dxd)


def test_half_steps():
    for t, h in HALF.items():
        assert h == torch.finfo(t).eps / 2

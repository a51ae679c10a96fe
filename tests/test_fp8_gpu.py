"""The linear layer in 8-bit floating point on the GPU: codes and scales bit for bit, products and gradients against 64 bits with
bounds that count roundings (oracle.fp8_block)."""
import numpy as np
import pytest
import torch

from oracle import fp8_block as fb

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
NAMES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
U = 2.0 ** -24


def rows_of(t, stride=None, offset=0, fill=float("nan")):
    """t on the GPU with a row stride and an offset into its memory (elements); the rest holds `fill`."""
    n, c = t.shape
    stride = c if stride is None else stride
    flat = torch.full((offset + n * stride + 8,), fill, dtype=t.dtype, device="cuda")
    v = flat[offset:offset + n * stride].view(n, stride)[:, :c]
    v.copy_(t)
    return v


def between(v, stride, offset):
    """What lies between the rows of rows_of()."""
    n, c = v.shape
    return v.as_strided((n, stride - c), (stride, 1), offset + c)


def hidden(rng, rows, C, dtype, size=1.0):
    x = rng.standard_normal((rows, C)).astype(np.float32) * np.exp(0.5 * rng.standard_normal((rows, 1))).astype(np.float32) * np.float32(size)
    x[:, rng.integers(0, C)] *= 20.0
    if rows > 3:
        x[rows // 2] = 0.0                  # padding
    if rows > 1:
        x[1, :130] = 0.0                    # a group without a value
        x[1, 140:] *= np.float32(1e-38)     # values near the end of the range (zero in fp16)
    return torch.from_numpy(x).to(NAMES[dtype])


def f64(t):
    return t.double().cpu().numpy()


def weights(rng, O, C):
    w = (rng.standard_normal((O, C)) * 0.05).astype(np.float32)
    w[rng.integers(0, O)] *= 8.0
    return w


def given(rng, O, C):
    """A checkpoint's weights: any codes but NaN, any scales."""
    codes = rng.integers(0, 256, (O, C)).astype(np.uint8)
    codes[(codes & 127) == 127] = 0
    scales = (np.exp(rng.standard_normal((-(-O // 128), -(-C // 128)))) * 1e-3).astype(np.float32)
    return codes, scales


def bits(t):
    return t.clone(memory_format=torch.contiguous_format).view(-1).view(torch.uint8).cpu().numpy()


# rows, rows of the plan, Cin
ROWS = [(1, 1, 1), (1, 5, 128), (3, 3, 129), (5, 8, 100), (16, 16, 4096), (17, 40, 640), (33, 33, 257), (77, 77, 768), (130, 200, 1000), (7, 7, 8200)]


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("case", ROWS, ids=lambda c: "%dof%d_%d" % c)
def test_quantize_rows(wq, case, dtype):
    n, R, C = case
    print(case, dtype, flush=True)
    rng = np.random.default_rng(n * 37 + C)
    plan = wq.Fp8LinearPlan(R, C, 8)
    x = hidden(rng, n, C, dtype)
    codes, scales = fb.quantize_rows(f64(x))
    for stride, off in ((C, 0), (C + 16, 16), (C + 5, 3)):
        ws = plan.alloc_workspace()
        ws.fill_(0xA5)
        before = [bits(v[n:]).tobytes() for v in plan.workspace_views(ws)]
        plan.quantize_rows(rows_of(x, stride, off), ws)
        torch.cuda.synchronize()
        got, s = plan.workspace_views(ws)
        assert np.array_equal(bits(got[:n]).reshape(n, -1) & 127, codes & 127)
        assert np.array_equal(f64(got[:n].float()), fb.decode(codes).reshape(n, -1))
        assert np.array_equal(f64(s[:n]), scales)
        assert before == [bits(v[n:]).tobytes() for v in plan.workspace_views(ws)]   # rows behind the last one stay


def test_codes_at_the_borders(wq):
    """Every middle between two codes, both ends of the scale's steps, and what is not a number."""
    v = fb.e4m3_values()
    mid = (v[1:] + v[:-1]) / 2
    x = np.zeros((6, 384), np.float32)
    x[0, :126], x[0, 126] = mid, 448.0
    x[1, :126], x[1, 126] = -np.nextafter(mid.astype(np.float32), np.float32(1e9)), 448.0
    x[2, 0], x[2, 130], x[2, 260] = 448.0, np.nextafter(np.float32(448), np.float32(1e9)), 3.3e38
    x[3, 0], x[3, 130], x[3, 260] = 1e-45, 2.0 ** -118, 1.0
    x[4, :] = 1.5
    x[4, 3], x[4, 200] = np.nan, np.inf
    x[5, 5], x[5, 140] = -np.inf, -3.4e38
    plan = wq.Fp8LinearPlan(6, 384, 8)
    ws = plan.alloc_workspace()
    plan.quantize_rows(torch.from_numpy(x).cuda(), ws)
    got, s = plan.workspace_views(ws)
    codes, scales = fb.quantize_rows(x)
    assert np.array_equal(f64(s), scales)
    assert np.array_equal(f64(got.float()), fb.decode(codes), equal_nan=True)


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("O,C", [(1, 1), (40, 200), (128, 128), (130, 384), (300, 1000), (2048, 16)])
def test_weight_prepare(wq, O, C, dtype):
    print(O, C, dtype, flush=True)
    rng = np.random.default_rng(O + C)
    w = torch.from_numpy(weights(rng, O, C)).to(NAMES[dtype])
    b = rng.standard_normal(O).astype(np.float32)
    codes, scales = fb.quantize_blocks(f64(w))
    for backward in (False, True):
        plan = wq.Fp8LinearPlan(4, C, O, backward=backward)
        blob = plan.alloc_blob()
        blob.fill_(0xFF)
        plan.weight_prepare(rows_of(w, C + 3, 1), torch.from_numpy(b).cuda(), blob)
        got, s, bias = plan.blob_views(blob)
        assert np.array_equal(f64(got.float()), fb.decode(codes)) and np.array_equal(f64(s), scales) and np.array_equal(bias.cpu().numpy(), b)
        if backward:
            L = plan.layout
            R, B = (C + 15) // 16 * 16, L.out_blocks
            t = blob[L.blob_codes_t_off:L.blob_codes_t_off + R * B * 128].view(torch.float8_e4m3fn).view(R // 16, B * 8, 16, 16).permute(0, 2, 1, 3)
            t = f64(t.reshape(R, B * 128).float())
            want = np.zeros_like(t)
            want[:C, :O] = fb.decode(codes).T
            assert np.array_equal(t, want)
            ts = blob[L.blob_scales_t_off:L.blob_scales_t_off + 4 * B * L.in_blocks].view(torch.float32).view(L.in_blocks, B)
            assert np.array_equal(f64(ts), scales.T)


def test_weight_load(wq):
    rng = np.random.default_rng(5)
    O, C = 300, 200
    codes, scales = given(rng, O, C)
    dev = torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn)
    plan = wq.Fp8LinearPlan(4, C, O, fp32_scales=True)
    blob = plan.alloc_blob()
    plan.weight_load(dev, torch.from_numpy(scales).cuda(), None, blob)
    got, s, bias = plan.blob_views(blob)
    assert np.array_equal(bits(got).reshape(O, C), codes) and np.array_equal(s.cpu().numpy(), scales) and not bias.any()
    e = torch.tensor([[0, 100], [127, 254], [255, 1]], dtype=torch.uint8)
    for p in (plan, wq.Fp8LinearPlan(4, C, O)):
        blob = p.alloc_blob()
        p.weight_load(dev, e.cuda().view(torch.float8_e8m0fnu), None, blob)
        _, s, _ = p.blob_views(blob)
        assert np.array_equal(f64(s), 2.0 ** (np.clip(e.numpy().astype(float), 1, 254) - 127))
    with pytest.raises(wq.WqError) as err:
        wq.Fp8LinearPlan(4, C, O).weight_load(dev, torch.from_numpy(scales).cuda(), None, blob)
    assert err.value.status == 2
    for bad in (lambda: plan.weight_load(dev.view(torch.uint8), torch.from_numpy(scales).cuda(), None, blob),
                lambda: plan.weight_load(dev, torch.from_numpy(scales).cuda().half(), None, blob),
                lambda: plan.weight_load(dev, torch.from_numpy(scales).cuda().t(), None, blob),
                lambda: plan.weight_load(dev[:10], torch.from_numpy(scales).cuda(), None, blob)):
        with pytest.raises(TypeError):
            bad()


def layer(wq, rng, R, C, O, loaded, backward=False, bias=True):
    """(plan, blob, workspace, the weights' values in 64 bits, bias)"""
    plan = wq.Fp8LinearPlan(R, C, O, backward=backward, fp32_scales=loaded)
    b = rng.standard_normal(O).astype(np.float32) if bias else None
    bd = None if b is None else torch.from_numpy(b).cuda()
    blob, ws = plan.alloc_blob(), plan.alloc_workspace()
    blob.fill_(0xFF)   # NaN codes and scales where nothing is written
    ws.fill_(0xFF)
    if loaded:
        codes, scales = given(rng, O, C)
        plan.weight_load(torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn), torch.from_numpy(scales).cuda(), bd, blob)
    else:
        w = weights(rng, O, C)
        codes, scales = fb.quantize_blocks(w)
        plan.weight_prepare(torch.from_numpy(w).cuda(), bd, blob)
    return plan, blob, ws, fb.block_values(codes, scales), b


def through_activation(e, z, act):
    """An error e of z behind the activation, and the activation's own (oracle.linear_block.epilogue_bound has the proof)."""
    return e if act in ("none", "relu") else 1.13 * e + 16 * U * (np.abs(fb.activation(z, act)) + 1.0)


def check(got, want, e):
    """|got - want| <= e and the type's own rounding (below its normal numbers half a spacing, an absolute amount)."""
    half = HALF[got.dtype]
    bound = e * 1.01 + half * (np.abs(want) + e) + torch.finfo(got.dtype).smallest_normal * half
    y = f64(got)
    bad = ~(np.abs(y - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(), float((np.abs(y - want) / bound)[~np.isnan(y)].max()))


# rows, rows of the plan, Cin, Cout, activation, gated, residual
PRODUCTS = [
    (1, 1, 1, 1, "none", False, False),
    (1, 1, 4096, 256, "none", False, True),
    (1, 7, 2048, 512, "silu", True, False),
    (2, 2, 512, 40, "relu", False, True),
    (3, 16, 200, 192, "gelu", True, True),
    (5, 5, 1024, 33, "gelu_tanh", False, False),
    (15, 40, 640, 576, "silu", True, True),
    (16, 16, 5000, 128, "none", False, False),
    (17, 17, 768, 100, "gelu", False, True),
    (31, 64, 1280, 320, "relu", True, False),
    (33, 64, 1280, 320, "relu", True, False),
    (63, 63, 896, 130, "silu", False, False),
    (77, 77, 768, 2040, "gelu_tanh", False, False),
    (129, 129, 500, 257, "none", False, True),
    (200, 300, 1536, 1088, "gelu", True, False),
    (257, 257, 256, 448, "silu", True, True),
    (1001, 1001, 2112, 136, "none", False, True),
    (520, 520, 384, 1504, "gelu_tanh", False, False),
    (1030, 1030, 640, 1280, "silu", False, True),
    (2050, 2050, 128, 96, "none", False, False),
    (4100, 4100, 64, 64, "relu", True, True),
    (260, 260, 130, 4160, "none", True, False),
    (300, 300, 127, 2900, "silu", False, True),
]


@pytest.mark.parametrize("loaded", [False, True], ids=["pow2", "any"])
@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("case", PRODUCTS, ids=lambda c: "%dof%d_%d-%d_%s_%d%d" % c)
def test_linear(wq, case, dtype, loaded):
    """linear() over strided tensors, then matmul() of the codes that quantize_rows leaves, with and without the values before the
    activation."""
    n, R, C, O, act, gated, with_res = case
    print(case, dtype, loaded, flush=True)
    rng = np.random.default_rng(n * 31 + C + O)
    plan, blob, ws, w, b = layer(wq, rng, R, C, O, loaded, bias=n % 3 != 0)
    outs = O // 2 if gated else O
    x = hidden(rng, n, C, dtype)
    res = torch.from_numpy(rng.standard_normal((n, outs)).astype(np.float32)).to(NAMES[dtype]) if with_res else None
    z, S = fb.product(fb.through(f64(x)), w, b)
    want = fb.epilogue(z, act, gated, None if res is None else f64(res))
    # the sum of Cin exact products, some partial sums and the bias: a rounding of the magnitudes' sum for each
    e = (C + 16) * U * S
    if gated:
        F = outs
        g, u = fb.activation(z[:, :F], act), z[:, F:]
        eg = through_activation(e[:, :F], z[:, :F], act)
        ey = np.abs(g) * e[:, F:] + np.abs(u) * eg + eg * e[:, F:] + U * np.abs(g * u)
    else:
        ey = through_activation(e, z, act)
    ey = ey + (U * np.abs(want) if with_res else 0)
    for k, (pad, off) in enumerate(((0, 0), (16, 8), (3, 1))):
        xd, rd = rows_of(x, C + pad, off), None if res is None else rows_of(res, outs + pad, off)
        y = rows_of(torch.zeros((n, outs), dtype=x.dtype), outs + pad, off)
        pre = rows_of(torch.zeros((n, O), dtype=x.dtype), O + pad, off) if k != 1 else None
        if k == 1 and res is not None:
            y = rd                               # in place
        if k == 2:
            plan.quantize_rows(xd, ws)
            plan.matmul(ws, blob, y, activation=act, gated=gated, residual=rd, preactivation=pre)
        else:
            plan.linear(xd, blob, ws, y, activation=act, gated=gated, residual=rd, preactivation=pre)
        torch.cuda.synchronize()
        check(y, want, ey)
        if pre is not None:
            check(pre, z, e)
            assert bool(between(pre, O + pad, off).isnan().all())
        if pad:
            assert bool(between(y, outs + pad, off).isnan().all())
        if dtype == "fp32" and act == "none" and not gated and n * O > 1000 and res is None:
            # sums keep their 24 bits: the matrix core's direct sums of codes are 1.5e-5 off.  Roundings of either sign, no more than a
            # partial sum of eight products each: sqrt(Cin / 8) half steps of what the terms add up to in the root mean square
            err = np.sqrt(np.mean((f64(y) - want) ** 2) / np.mean(want ** 2))
            assert err <= (np.sqrt(C / 8) + 4) * U, err


# rows, rows of the plan, Cin, Cout, activation, gated, dw in fp32
GRADS = [
    (1, 1, 1, 1, "none", False, True),
    (1, 4, 300, 200, "none", False, True),
    (3, 3, 128, 128, "silu", False, False),
    (16, 16, 640, 320, "gelu", True, False),
    (33, 33, 257, 130, "none", False, True),
    (127, 128, 512, 384, "relu", False, False),
    (128, 128, 100, 64, "silu", True, True),
    (129, 200, 384, 1024, "gelu_tanh", True, False),
    (300, 300, 768, 500, "none", False, False),
    (1000, 1000, 200, 320, "gelu", True, False),
    (1500, 1500, 130, 140, "none", False, True),
    (2100, 2100, 96, 72, "relu", False, True),
    (520, 520, 1100, 1300, "none", False, True),
    (640, 640, 1280, 1152, "silu", True, False),
]


def uncertain(v, delta, axis):
    """How far apart the values of the codes are for v a little larger and a little smaller: not zero next to a border."""
    q = (lambda t: fb.through(t)) if axis == 1 else (lambda t: fb.through(t.T).T)
    return np.abs(q(v + delta) - q(v - delta))


@pytest.mark.parametrize("loaded", [False, True], ids=["pow2", "any"])
@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("case", GRADS, ids=lambda c: "%dof%d_%d-%d_%s_%d%d" % c)
def test_backward(wq, case, dtype, loaded):
    n, R, C, O, act, gated, wide = case
    print(case, dtype, loaded, flush=True)
    rng = np.random.default_rng(n * 17 + C + O)
    plan, blob, ws, w, _ = layer(wq, rng, R, C, O, loaded, backward=True)
    outs, T = O // 2 if gated else O, NAMES[dtype]
    x, dy = hidden(rng, n, C, dtype), hidden(rng, n, outs, dtype, 1e-2)
    through = act != "none" or gated
    pre = torch.from_numpy((1.5 * rng.standard_normal((n, O))).astype(np.float32)).to(T) if through else None
    dz = fb.gate_grad(f64(dy), f64(pre) if through else None, act, gated)
    # dz in fp32: the slope is a sum of two terms of up to some units in size, each off by a few roundings, as is the value
    d64 = np.abs(f64(dy))
    if not through:
        delta = np.zeros_like(dz)
    elif gated:
        g, u = f64(pre)[:, :outs], f64(pre)[:, outs:]
        delta = np.concatenate([d64 * np.abs(u) * (np.abs(fb.slope(g, act)) + 1) * 16 * U, d64 * (np.abs(fb.activation(g, act)) + 1) * 16 * U], 1)
    else:
        delta = d64 * (np.abs(fb.slope(f64(pre), act)) + 1) * 16 * U
    D1, D2, X2 = fb.through(dz), fb.through(dz.T).T, fb.through(f64(x).T).T
    direct = 7 * 2.0 ** -13   # of eight products up to seven are cut off at 2^-13 of the largest
    Sx, Sw = np.abs(D1) @ np.abs(w), np.abs(D2).T @ np.abs(X2)
    ex = (O + 16) * U * Sx + uncertain(dz, delta, 1) @ np.abs(w) + (direct * Sx if dtype != "fp32" else 0)
    fp32_w = wide or dtype == "fp32"
    ew = (n + 16) * U * Sw + uncertain(dz, delta, 0).T @ np.abs(X2) + (0 if fp32_w else direct * Sw)
    eb = (n + 4) * U * np.abs(dz).sum(0) + delta.sum(0)
    want_x, want_w, want_b = D1 @ w, D2.T @ X2, dz.sum(0)
    for k, (pad, off) in enumerate(((0, 0), (16, 8), (3, 1))):
        xd, dyd = rows_of(x, C + pad, off), rows_of(dy, outs + pad, off)
        pd = rows_of(pre, O + pad, off) if through else None
        dx = xd if k == 1 else rows_of(torch.zeros((n, C), dtype=T), C + pad, off)
        dw = rows_of(torch.zeros((O, C), dtype=torch.float32 if fp32_w else T), C + pad, off)
        db = torch.full((O,), float("nan"), device="cuda")
        ws.fill_(0xFF)
        plan.backward(xd, dyd, blob, ws, dx=dx, dw=dw, db=db, preactivation=pd, activation=act, gated=gated)
        torch.cuda.synchronize()
        check(dx, want_x, ex)
        check(dw, want_w, ew)
        check(db, want_b, eb)
        if pad:
            assert bool(between(dx, C + pad, off).isnan().all()) and bool(between(dw, C + pad, off).isnan().all())
        if n * O > 5000 and not through:   # no more than the type's rounding, in the root mean square
            for got, want in ((dx, want_x), (dw, want_w)):
                rel = np.sqrt(((f64(got) - want) ** 2).sum() / (want ** 2).sum())
                assert rel <= (1e-5 if got.dtype == torch.float32 else HALF[got.dtype] * 0.75), rel
        if k == 0:   # the same bits again, and added to what is there
            dx2, dw2, db2 = torch.empty_like(dx), torch.empty_like(dw), torch.empty_like(db)
            plan.backward(xd, dyd, blob, ws, dx=dx2, dw=dw2, db=db2, preactivation=pd, activation=act, gated=gated)
            assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)
            plan.backward(xd, dyd, blob, ws, dw=dw2, db=db2, preactivation=pd, activation=act, gated=gated, accumulate=True)
            check(dw2, want_w + f64(dw), ew + U * np.abs(2 * want_w))
            check(db2, want_b + f64(db), eb + U * np.abs(2 * want_b))
            # one at a time
            only = torch.empty_like(dx)
            plan.backward(None, dyd, blob, ws, dx=only, preactivation=pd, activation=act, gated=gated)
            assert torch.equal(only, dx)
            only = torch.empty_like(dw)
            plan.backward(xd, dyd, None, ws, dw=only, preactivation=pd, activation=act, gated=gated)
            assert torch.equal(only, dw)
            only = torch.empty_like(db)
            plan.backward(None, dyd, None, ws, db=only, preactivation=pd, activation=act, gated=gated)
            assert torch.equal(only, db)


def test_gradients_against_differences(wq):
    """A loss of the layer itself, moved along a direction: its weights' and inputs' codes stay what they are where a change is
    a whole number of their steps, so the difference is the product's own."""
    rng = np.random.default_rng(9)
    n, C, O = 40, 256, 128
    plan, blob, ws, w, _ = layer(wq, rng, n, C, O, False, backward=True, bias=False)
    base = rng.choice(np.arange(16, 32), (n, C)).astype(np.float32) * rng.choice([-1.0, 1.0], (n, C)).astype(np.float32)
    base[:, ::128] = 448.0   # every group's scale is 1: whole numbers up to 32 are codes, up to 16 all of them in steps of 1
    step = np.where(np.abs(base) < 32, 2.0, 0.0).astype(np.float32) * np.sign(base)
    lo, hi = np.where(step != 0, np.trunc(base / 4) * 4, base), None
    hi = np.where(step != 0, lo + 4 * np.sign(base), base)
    dy = rng.choice([-1.0, 0.5, 2.0], (n, O)).astype(np.float32)
    loss = []
    for x in (lo, hi):
        y = torch.empty(n, O, device="cuda")
        plan.linear(torch.from_numpy(x).cuda(), blob, ws, y)
        loss.append((f64(y) * dy).sum())
    dx = torch.empty(n, C, device="cuda")
    plan.backward(None, torch.from_numpy(dy).cuda(), blob, ws, dx=dx)
    moved = (f64(dx) * (hi - lo).astype(np.float64)).sum()
    size = np.abs(dy).sum() * 448 * np.abs(w).sum(1).max()
    assert abs((loss[1] - loss[0]) - moved) <= 2 * (C + 16) * U * size


def test_no_rows(wq):
    rng = np.random.default_rng(3)
    plan, blob, ws, _, _ = layer(wq, rng, 4, 200, 64, False, backward=True)
    empty = torch.empty((0, 200), device="cuda", dtype=torch.bfloat16)
    y = torch.empty((0, 64), device="cuda", dtype=torch.bfloat16)
    plan.linear(empty, blob, ws, y)
    plan.quantize_rows(empty, ws)
    plan.layer_norm_quantize(empty, ws)
    for wt in (torch.float32, torch.bfloat16):
        dw, db = torch.ones((64, 200), device="cuda", dtype=wt), torch.ones(64, device="cuda")
        plan.backward(empty, y, blob, ws, dx=torch.empty_like(empty), dw=dw, db=db, accumulate=True)
        assert bool((dw == 1).all()) and bool((db == 1).all())
        plan.backward(empty, y, blob, ws, dx=torch.empty_like(empty), dw=dw, db=db)
        assert not dw.any() and not db.any()


def test_infinities_and_nan_stay_in_their_rows(wq):
    rng = np.random.default_rng(4)
    for n in (4, 40, 300):
        plan, blob, ws, w, b = layer(wq, rng, n, 300, 256, False, backward=True)
        x = torch.from_numpy(rng.standard_normal((n, 300)).astype(np.float32)).bfloat16()
        x[1, 7], x[2, 200] = float("nan"), float("inf")
        y = torch.empty((n, 256), device="cuda", dtype=torch.bfloat16)
        plan.linear(x.cuda(), blob, ws, y)
        assert bool(y[1:3].isnan().all()) and not bool(y[0].isnan().any()) and not bool(y[3:].isnan().any())
        dx, dw, db = torch.empty((n, 300), device="cuda", dtype=torch.bfloat16), torch.empty((256, 300), device="cuda"), torch.empty(256, device="cuda")
        dy = torch.ones((n, 256), device="cuda", dtype=torch.bfloat16)
        dy[2, 5] = float("nan")
        plan.backward(x.cuda(), dy, blob, ws, dx=dx, dw=dw, db=db)
        assert bool(dx[2].isnan().all()) and int(dx.isnan().sum()) == 300
        nan = dw.isnan()
        assert bool(nan[5].all()) and bool(nan[:, 7].all()) and bool(nan[:, 200].all()) and int(nan.sum()) == 300 + 2 * 255
        assert bool(db[5].isnan()) and int(db.isnan().sum()) == 1


def test_two_streams_with_a_workspace_each(wq):
    rng = np.random.default_rng(6)
    plan, blob, ws, w, b = layer(wq, rng, 64, 512, 640, False, backward=True)
    xs = [hidden(rng, 64, 512, "bf16").cuda() for _ in range(2)]
    want = []
    for x in xs:
        y, dw = torch.empty((64, 640), device="cuda", dtype=x.dtype), torch.empty((640, 512), device="cuda")
        plan.linear(x, blob, ws, y)
        plan.backward(x, y, blob, ws, dw=dw)
        want.append((y, dw))
    torch.cuda.synchronize()
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [ws, plan.alloc_workspace()]
    got = [(torch.empty_like(y), torch.empty_like(dw)) for y, dw in want]
    torch.cuda.synchronize()
    for _ in range(5):
        for k in range(2):
            plan.linear(xs[k], blob, spaces[k], got[k][0], stream=streams[k])
            plan.backward(xs[k], got[k][0], blob, spaces[k], dw=got[k][1], stream=streams[k])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


class Block:
    """A feed-forward block over a residual stream, forward and backward: norm, gated projection, projection back."""

    def __init__(self, wq, rng, rows, C, F, act="silu"):
        self.act = act
        self.norm = wq.LayerNormPlan(rows, C)
        self.up, self.up_blob, self.up_ws, self.w1, self.b1 = layer(wq, rng, rows, C, 2 * F, False, backward=True)
        self.down, self.down_blob, self.down_ws, self.w2, self.b2 = layer(wq, rng, rows, F, C, False, backward=True)
        self.norm_ws = self.norm.alloc_workspace()
        self.gamma = torch.from_numpy((1 + 0.2 * rng.standard_normal(C)).astype(np.float32)).cuda()
        self.beta = torch.from_numpy((0.1 * rng.standard_normal(C)).astype(np.float32)).cuda()
        new = lambda *s: torch.empty(s, device="cuda")   # noqa: E731
        low = lambda *s: torch.empty(s, device="cuda", dtype=torch.bfloat16)   # noqa: E731
        self.h, self.y, self.pre, self.mid, self.out = low(rows, C), low(rows, C), low(rows, 2 * F), low(rows, F), low(rows, C)
        self.dmid, self.dy, self.dx = low(rows, F), low(rows, C), low(rows, C)
        self.dw1, self.dw2, self.db1, self.db2 = new(2 * F, C), new(C, F), new(2 * F), new(C)
        self.dgamma, self.dbeta = new(C), new(C)

    def forward(self, x, res):
        self.norm.forward(x, self.y, gamma=self.gamma, beta=self.beta, residual=res, out=self.h)
        self.up.linear(self.y, self.up_blob, self.up_ws, self.mid, activation=self.act, gated=True, preactivation=self.pre)
        self.down.linear(self.mid, self.down_blob, self.down_ws, self.out, residual=self.h)

    def backward(self, dout):
        self.down.backward(self.mid, dout, self.down_blob, self.down_ws, dx=self.dmid, dw=self.dw2, db=self.db2)
        self.up.backward(self.y, self.dmid, self.up_blob, self.up_ws, dx=self.dy, dw=self.dw1, db=self.db1, preactivation=self.pre,
                         activation=self.act, gated=True)
        self.norm.backward(self.dy, self.h, self.norm_ws, dx=self.dx, gamma=self.gamma, residual_grad=dout, dgamma=self.dgamma, dbeta=self.dbeta)

    def results(self):
        return [self.out, self.dx, self.dw1, self.dw2, self.db1, self.db2, self.dgamma, self.dbeta]


def test_a_block_forward_and_backward(wq):
    """The operators in a run, each against its formula on what the one before left."""
    rng = np.random.default_rng(11)
    n, C, F = 150, 320, 448
    B = Block(wq, rng, n, C, F)
    x, res, dout = (hidden(rng, n, C, "bf16").cuda() for _ in range(3))
    B.forward(x, res)
    B.backward(dout)
    torch.cuda.synchronize()
    h, v = fb.layer_norm(f64(x), f64(res), B.gamma.cpu().numpy(), B.beta.cpu().numpy(), 1e-5)
    assert torch.equal(B.h.cpu(), torch.from_numpy(h).bfloat16())
    z, S = fb.product(fb.through(f64(B.y)), B.w1, B.b1)
    check(B.pre, z, (C + 16) * U * S)
    z, S = fb.product(fb.through(f64(B.mid)), B.w2, B.b2)
    check(B.out, z + f64(B.h), (F + 17) * U * (S + np.abs(f64(B.h))))
    D = fb.through(f64(dout))
    check(B.dmid, D @ B.w2, 7 * 2.0 ** -13 * np.abs(D) @ np.abs(B.w2))
    dx, dgamma, dbeta = fb.layer_norm_grad(f64(B.dy), f64(B.h), B.gamma.cpu().numpy(), f64(dout), 1e-5)
    for got, want in ((B.dx, dx), (B.dgamma, dgamma), (B.dbeta, dbeta)):
        rel = np.sqrt(((f64(got) - want) ** 2).sum() / (want ** 2).sum())
        assert rel <= (2e-6 if got.dtype == torch.float32 else 2.0 ** -8 * 0.75), rel


def test_a_captured_block(wq):
    """A training step in a graph, replayed on new inputs with eager work between the replays, gives the eager step's bits."""
    rng = np.random.default_rng(12)
    n, C, F = 200, 256, 384
    B = Block(wq, rng, n, C, F)
    sets = [[hidden(rng, n, C, "bf16").cuda() for _ in range(3)] for _ in range(3)]
    want = []
    for x, res, dout in sets:
        B.forward(x, res)
        B.backward(dout)
        want.append([t.clone() for t in B.results()])
    ins = [torch.empty_like(t) for t in sets[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.forward(ins[0], ins[1])
        B.backward(ins[2])
    for k in (0, 1, 2, 1, 0):
        for a, b in zip(ins, sets[k]):
            a.copy_(b)
        for t in B.results():
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(B.results(), want[k]))
        B.forward(*sets[(k + 1) % 3][:2])   # the program's own work between
        B.backward(sets[(k + 1) % 3][2])


def test_rows_far_apart(wq):
    """Rows 2^27 elements apart: offsets beyond 32 bits."""
    rng = np.random.default_rng(13)
    n, C, O, stride = 9, 128, 64, 1 << 27
    plan, blob, ws, w, b = layer(wq, rng, n, C, O, False, backward=True)
    big = torch.empty((n * stride,), dtype=torch.bfloat16, device="cuda").view(n, stride)
    x = hidden(rng, n, C, "bf16")
    xd, yd, dyd, dxd = big[:, :C], big[:, 200:200 + O], big[:, 400:400 + O], big[:, 600:600 + C]
    xd.copy_(x)
    dyd.copy_(hidden(rng, n, O, "bf16"))
    plan.linear(xd, blob, ws, yd)
    z, S = fb.product(fb.through(f64(x)), w, b)
    check(yd, z, (C + 16) * U * S)
    dw = torch.empty((O, C), device="cuda")
    plan.backward(xd, dyd, blob, ws, dx=dxd, dw=dw)
    D = fb.through(f64(dyd))
    check(dxd, D @ w, 7 * 2.0 ** -13 * np.abs(D) @ np.abs(w))
    D2, X2 = fb.through(f64(dyd).T).T, fb.through(f64(x).T).T
    check(dw, D2.T @ X2, (n + 16) * U * np.abs(D2).T @ np.abs(X2))


def test_binding_refusals(wq):
    plan = wq.Fp8LinearPlan(4, 200, 128, backward=True)
    blob, ws = plan.alloc_blob(), plan.alloc_workspace()
    x, y, dw = (torch.zeros(s, device="cuda", dtype=torch.bfloat16) for s in ((4, 200), (4, 128), (128, 200)))
    plan.weight_prepare(dw, None, blob)
    for f in (lambda: plan.linear(x, blob, ws, y.float()), lambda: plan.linear(x, blob, ws, None), lambda: plan.linear(x, ws.int(), ws, y),
              lambda: plan.backward(x, y, blob, ws, dw=dw.half()), lambda: plan.backward(x, y, blob, ws, db=torch.zeros(128).cuda().half()),
              lambda: plan.layer_norm_quantize(x, ws, gamma=dw), lambda: plan.weight_prepare(dw, dw, blob)):
        with pytest.raises(TypeError):
            f()
    for f in (lambda: plan.linear(x[:, :100], blob, ws, y), lambda: plan.linear(x, blob, ws, y[:2]), lambda: plan.linear(x, blob, ws, y, preactivation=x),
              lambda: plan.linear(x, blob, ws, y, gated=True), lambda: plan.backward(x, y, blob, ws, dx=y), lambda: plan.backward(x, y, blob, ws, dw=dw.t()),
              lambda: plan.layer_norm_quantize(x, ws, beta=torch.zeros(199).cuda()), lambda: plan.weight_prepare(dw[:5], None, blob),
              lambda: plan.quantize_rows(torch.zeros((5, 200), device="cuda"), ws), lambda: plan.quantize_rows(x.t(), ws)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(wq.WqError):
        plan.backward(x, y, blob, ws, dx=x, activation="silu")   # without the values before the activation
    with pytest.raises(wq.WqError):
        plan.backward(x, y, None, ws, dx=x)


@pytest.mark.parametrize("act", ["relu", "silu", "gelu", "gelu_tanh"])
def test_slopes_by_place(wq, act):
    """The bias's gradient of one row is dz itself: slopes and values over the whole range, at infinities and NaN."""
    z = np.concatenate([np.linspace(-14, 14, 3001), [-300.0, -40.0, 0.0, -0.0, 300.0, 6e4, np.inf, -np.inf, np.nan] * 8, np.zeros(63)])
    z = z[:len(z) // 64 * 64].astype(np.float32)
    n = len(z)
    lim = np.where(np.isinf(z), np.sign(z) * 1e4, z).astype(np.float64)
    slope, value = fb.slope(lim, act), fb.activation(lim, act)
    plan = wq.Fp8LinearPlan(1, 8, n, backward=True)
    ws = plan.alloc_workspace()
    db = torch.empty(n, device="cuda")
    plan.backward(None, torch.ones((1, n), device="cuda"), None, ws, db=db, preactivation=torch.from_numpy(z).cuda()[None], activation=act)
    nan = np.isnan(z)
    got = f64(db)
    # s and 1 - s, or the tail and the density, are each off by a few units relative to themselves and are added after a product with z
    tol = 16 * U * (1 + np.abs(lim) * (np.abs(lim) < 20))
    assert (np.abs(got - slope)[~nan] <= tol[~nan]).all() and np.isnan(got[nan]).all()
    # gated: the second half's gradient is the value of the first
    plan = wq.Fp8LinearPlan(1, 8, 2 * n, backward=True)
    ws = plan.alloc_workspace()
    db = torch.empty(2 * n, device="cuda")
    pre = torch.cat([torch.from_numpy(z), torch.full((n,), 0.5)])[None].cuda()
    plan.backward(None, torch.ones((1, n), device="cuda"), None, ws, db=db, preactivation=pre, activation=act, gated=True)
    got = f64(db)
    assert (np.abs(got[:n] - 0.5 * slope)[~nan] <= tol[~nan]).all()
    fine = np.isfinite(z)
    assert (np.abs(got[n:] - value)[fine] <= 16 * U * (np.abs(value) + 1)[fine]).all()
    assert (got[n:][z == np.inf] == np.inf).all() and not got[n:][z == -np.inf].any() and np.isnan(got[n:][nan]).all()

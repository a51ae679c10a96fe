"""The linear layer's surroundings on the GPU: norm with the residual's addition into codes, row quantization, and the
product with bias, activation, gate and residual, against the oracle in 64 bits.  Codes, scales and the
stored sum are compared bit for bit, products with a bound that counts roundings (oracle.linear_block)."""
import numpy as np
import pytest
import torch

import oracle
from oracle import linear_block as lb

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
NAMES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def rows_of(t, stride=None, offset=0, fill=float("nan")):
    """t on the GPU with a row stride and an offset into its memory (elements); the rest holds `fill`."""
    n, c = t.shape
    stride = c if stride is None else stride
    flat = torch.full((offset + n * stride + 8,), fill, dtype=t.dtype, device="cuda")
    v = flat[offset:offset + n * stride].view(n, stride)[:, :c]
    v.copy_(t)
    return v


def hidden(rng, rows, C, dtype):
    x = rng.standard_normal((rows, C)).astype(np.float32) * np.exp(0.5 * rng.standard_normal((rows, 1))).astype(np.float32)
    x[:, rng.integers(0, C)] *= 20.0
    if rows > 3:
        x[rows // 2] = 0.0                  # padding
    if rows > 1:
        x[1, :32] = 0.0                     # a group without a value
        x[1, 40:] *= np.float32(1e-38)      # values near the end of the range (zero in fp16)
    return torch.from_numpy(x).to(NAMES[dtype])


def f32(t):
    return t.float().cpu().numpy()


def check_codes(plan, ws, n, codes, scales):
    xq, sx = plan.workspace_views(ws)
    assert np.array_equal(xq[:n].cpu().numpy(), codes)
    assert np.array_equal(sx[:n].cpu().numpy().view(np.uint32), scales.view(np.uint32))


# rows, rows of the plan, Cin, g
NORMS = [(1, 1, 32, 32), (1, 5, 64, 64), (3, 3, 512, 512), (5, 8, 96, 32), (7, 7, 640, 128), (16, 16, 4096, 128), (9, 33, 1280, 64),
         (130, 130, 320, 64), (2, 2, 8192, 256), (17, 17, 5120, 512), (3, 3, 16384, 64), (2, 4, 33280, 512), (1, 1, 65536, 32),
         (1, 16, 4096, 128), (65, 65, 2016, 32)]


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("case", NORMS, ids=lambda c: "%dof%d_%d_g%d" % c)
def test_rms_norm_quantize(wq, case, dtype):
    n, R, C, g = case
    print(case, dtype, flush=True)
    rng = np.random.default_rng(n * 131 + C)
    plan = wq.LinearPlan(R, C, 32, g)
    x, res = hidden(rng, n, C, dtype), hidden(rng, n, C, dtype)
    gamma = (1.0 + 0.2 * rng.standard_normal(C)).astype(np.float32)
    for with_res, with_gamma, strided, sum_into in ((1, 1, 0, "out"), (0, 0, 0, None), (1, 0, 1, "residual"), (1, 1, 2, "x"), (0, 1, 1, "out")):
        ws = plan.alloc_workspace()
        ws.fill_(0xA5)
        before = [v[n:].cpu().numpy().tobytes() for v in plan.workspace_views(ws)]
        # 1: a row stride of whole 16-byte pieces, 2: odd strides and offsets
        stride, off = ((C, 0), (C + 16, 8), (C + 3, 1))[strided]
        xd, rd = rows_of(x, stride, off), rows_of(res, stride, off) if with_res else None
        out = {"out": rows_of(torch.zeros_like(x), stride, off), "residual": rd, "x": xd, None: None}[sum_into]
        gd = torch.from_numpy(gamma).cuda() if with_gamma else None
        plan.rms_norm_quantize(xd, ws, residual=rd, gamma=gd, eps=1e-5, out=out)
        torch.cuda.synchronize()
        h, codes, scales = lb.rms_norm_quantize(f32(x), f32(res) if with_res else None, gamma if with_gamma else None, 1e-5, g)
        check_codes(plan, ws, n, codes, scales)
        if out is not None:
            assert torch.equal(out.cpu(), torch.from_numpy(h).to(x.dtype))
            beyond = out.as_strided((n, stride - C), (stride, 1), off + C)   # what lies between the rows
            assert bool(beyond.isnan().all())
        # rows behind the last one stay
        assert before == [v[n:].cpu().numpy().tobytes() for v in plan.workspace_views(ws)]


def test_rms_norm_of_extreme_rows(wq):
    """Sums of squares beyond fp32, one value in a row of zeros, rows of one tiny value."""
    C, g = 256, 64
    x = torch.zeros(6, C)
    x[0] = 1e30
    x[1, 7] = -3e38
    x[2] = 1e-30
    x[3, 255] = 1e-20
    x[4] = torch.linspace(-1, 1, C)
    plan = wq.LinearPlan(6, C, 32, g)
    ws = plan.alloc_workspace()
    for eps in (1e-6, 2.0 ** -126, 1e30):
        plan.rms_norm_quantize(x.cuda(), ws, eps=eps)
        torch.cuda.synchronize()
        _, codes, scales = lb.rms_norm_quantize(x.numpy(), None, None, eps, g)
        check_codes(plan, ws, 6, codes, scales)


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("case", NORMS, ids=lambda c: "%dof%d_%d_g%d" % c)
def test_quantize_rows(wq, case, dtype):
    n, R, C, g = case
    print(case, dtype, flush=True)
    rng = np.random.default_rng(n * 37 + C)
    plan = wq.LinearPlan(R, C, 32, g)
    x = hidden(rng, n, C, dtype)
    codes, scales = oracle.quantize_pixels(f32(x), g)
    for stride, off in ((C, 0), (C + 16, 16), (C + 5, 3)):
        ws = plan.alloc_workspace()
        plan.quantize_rows(rows_of(x, stride, off), ws)
        torch.cuda.synchronize()
        check_codes(plan, ws, n, codes, scales)


def layer(wq, rng, R, Cin, Cout, g, bits, bias=True):
    plan = wq.LinearPlan(R, Cin, Cout, g, weight_bits=bits)
    w = (rng.standard_normal((Cout, Cin)) * 0.05).astype(np.float32)
    b = rng.standard_normal(Cout).astype(np.float32) if bias else None
    blob, ws = plan.alloc_blob(), plan.alloc_workspace()
    ws.fill_(0xFF)   # NaN scales where nothing is written
    plan.weight_prepare(torch.from_numpy(w).cuda(), None if b is None else torch.from_numpy(b).cuda(), blob)
    return plan, blob, ws, oracle.quantize_weight_rows(w, g, bits), b


def check_product(got, z, S, groups, act, gated, res):
    want = lb.epilogue(z, act, gated, res)
    # below the type's normal numbers its spacing is one and the same, so a rounding there is off by up to half of that in
    # absolute terms: fp16's numbers below 2^-14 are 2^-24 apart
    bound = lb.epilogue_bound(z, S, groups, act, gated, res, HALF[got.dtype]) + torch.finfo(got.dtype).smallest_normal * HALF[got.dtype]
    y = got.double().cpu().numpy()
    bad = ~(np.abs(y - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(), float((np.abs(y - want) / bound)[~np.isnan(y)].max()))


# rows, rows of the plan, Cin, Cout, g, activation, gated, residual
PRODUCTS = [
    (1, 1, 32, 1, 32, "none", False, False),
    (1, 1, 4096, 256, 128, "none", False, True),
    (1, 7, 2048, 512, 64, "silu", True, False),
    (2, 2, 512, 40, 512, "relu", False, True),
    (3, 16, 320, 96, 32, "gelu", True, True),
    (5, 5, 1024, 33, 256, "gelu_tanh", False, False),
    (15, 40, 640, 544, 128, "silu", True, True),
    (16, 16, 5120, 128, 64, "none", False, False),
    (17, 17, 768, 100, 32, "gelu", False, True),
    (33, 64, 1280, 320, 64, "relu", True, False),
    (63, 63, 896, 130, 128, "silu", False, False),
    (77, 77, 768, 2048, 32, "gelu_tanh", False, False),
    (129, 129, 512, 257, 64, "none", False, True),
    (200, 300, 1536, 1088, 512, "gelu", True, False),
    (257, 257, 256, 512, 256, "silu", True, True),
    (1001, 1001, 2048, 136, 128, "none", False, True),
    (520, 520, 384, 1504, 128, "gelu_tanh", True, False),
    (1030, 1030, 640, 1280, 64, "silu", False, True),
    (2050, 2050, 128, 96, 32, "none", False, False),
    (4100, 4100, 64, 64, 64, "relu", True, True),
    (16, 16, 512, 96, 64, "silu", True, True),
    (8, 9, 1024, 48, 256, "relu", False, False),
    (4, 4, 2048, 64, 512, "none", True, False),
    (16, 16, 512, 31, 32, "none", False, True),
    (16, 16, 1024, 64, 128, "gelu", True, False),   # the most that one launch quantizes and multiplies
    (4, 4, 4096, 80, 512, "none", False, True),
    (1, 1, 16384, 48, 64, "none", False, False),
    (16, 16, 1056, 64, 32, "none", False, False),   # a little more
    (50, 50, 768, 288, 32, "silu", True, True),     # several blocks of rows, each quantized by the workgroups that multiply it
    (100, 130, 1024, 150, 256, "none", False, False),
    (33, 33, 64, 1000, 64, "relu", False, True),
]

# every kernel form, at sizes well inside the rules that choose it: (rows, weight rows) and whether the reduction has to be long
FORMS = {"rows": (13, 96, False), "rows2": (101, 640, False), "teams4": (199, 2240, False), "teams2": (301, 4480, False),
         "teams1": (641, 4480, False), "large": (2501, 4480, True)}
SHORT = {32: 224, 64: 192, 128: 384, 256: 768, 512: 1536}   # 32, 64: the last stage of 128 bytes is not a whole one


@pytest.mark.parametrize("bits", [8, 4], ids=["w8", "w4"])
@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("case", PRODUCTS, ids=lambda c: "%dof%d_%d-%d_g%d_%s_%d%d" % c)
def test_linear(wq, case, dtype, bits):
    """linear() over strided tensors, then matmul() of the codes that quantize_rows leaves: both within the bound."""
    n, R, Cin, Cout, g, act, gated, with_res = case
    print(case, dtype, bits, flush=True)
    rng = np.random.default_rng(n * 31 + Cin + Cout)
    plan, blob, ws, (wcodes, wscales), b = layer(wq, rng, R, Cin, Cout, g, bits, bias=n % 3 != 0)
    outs = Cout // 2 if gated else Cout
    x = hidden(rng, n, Cin, dtype)
    res = torch.from_numpy(rng.standard_normal((n, outs)).astype(np.float32)).to(NAMES[dtype]) if with_res else None
    codes, scales = oracle.quantize_pixels(f32(x), g)
    z, S = lb.product(codes, scales, wcodes, wscales, b, g)
    for k, (pad, off) in enumerate(((0, 0), (16, 8), (3, 1))):
        xd, rd = rows_of(x, Cin + pad, off), None if res is None else rows_of(res, outs + pad, off)
        y = rows_of(torch.zeros((n, outs), dtype=NAMES[dtype]), outs + pad, off)
        if k == 1 and res is not None:
            y = rd                               # in place
        if k == 2:
            plan.quantize_rows(xd, ws)
            plan.matmul(ws, blob, y, activation=act, gated=gated, residual=rd)
        else:
            plan.linear(xd, blob, ws, y, activation=act, gated=gated, residual=rd)
        torch.cuda.synchronize()
        check_product(y, z, S, Cin // g, act, gated, None if res is None else f32(res))
        if pad:
            assert bool(y.as_strided((n, pad), (outs + pad, 1), off + outs).isnan().all())


@pytest.mark.parametrize("bits", [8, 4], ids=["w8", "w4"])
@pytest.mark.parametrize("g", SHORT)
@pytest.mark.parametrize("form", FORMS)
def test_every_form_of_the_product(wq, form, g, bits):
    """Each form with each group size, gated and not, with columns that nothing divides; the oracle on a sample of rows: the
    ends, both sides of every kind of tile border, and some between."""
    n, Cout, long_k = FORMS[form]
    print(form, g, bits, flush=True)
    rng = np.random.default_rng(g + bits)
    Cin = 2048 if long_k and g >= 128 else SHORT[g]
    for gated, less in ((True, 0), (False, 3)):
        plan, blob, ws, (wcodes, wscales), b = layer(wq, rng, n, Cin, Cout - less, g, bits)
        outs = Cout // 2 if gated else Cout - less
        x = hidden(rng, n, Cin, "bf16")
        y = torch.full((n, outs), float("nan"), dtype=torch.bfloat16, device="cuda")
        res = torch.from_numpy(rng.standard_normal((n, outs)).astype(np.float32)).bfloat16()
        plan.linear(x.cuda(), blob, ws, y, activation="silu", gated=gated, residual=res.cuda())
        torch.cuda.synchronize()
        assert bool(y.isfinite().all())
        rows = sorted({r for r in (0, 1, 15, 16, 31, 32, 63, 64, 127, 128, 255, 256, n // 2, n - 2, n - 1) if r < n} |
                      set(rng.integers(0, n, 12).tolist()))
        codes, scales = oracle.quantize_pixels(f32(x[rows]), g)
        z, S = lb.product(codes, scales, wcodes, wscales, b, g)
        check_product(y[torch.tensor(rows, device="cuda")], z, S, Cin // g, "silu", gated, f32(res[rows]))


def test_output_in_the_place_of_its_input(wq):
    """x + f(x) written over x: by one row, where the product would read x itself, and by many."""
    rng = np.random.default_rng(17)
    for n in (1, 6, 70):
        plan, blob, ws, (wcodes, wscales), b = layer(wq, rng, n, 512, 512, 64, 8)
        x = hidden(rng, n, 512, "fp32")
        z, S = lb.product(*oracle.quantize_pixels(f32(x), 64), wcodes, wscales, b, 64)
        xd = x.cuda()
        plan.linear(xd, blob, ws, xd, activation="gelu", residual=xd)
        torch.cuda.synchronize()
        check_product(xd, z, S, 8, "gelu", False, f32(x))


def test_two_streams_at_once(wq):
    """Calls on two streams with a workspace each, again and again without a wait between them: as if alone."""
    rng = np.random.default_rng(23)
    sides = []
    for n, Cin, Cout, g, bits in ((300, 1024, 768, 64, 4), (7, 1024, 512, 128, 8)):
        plan, blob, ws, _, _ = layer(wq, rng, n, Cin, Cout, g, bits)
        x = hidden(rng, n, Cin, "bf16").cuda()
        y = torch.empty((n, Cout), dtype=torch.bfloat16, device="cuda")
        h = torch.empty_like(x)
        plan.rms_norm_quantize(x, ws, residual=x, out=h)
        plan.matmul(ws, blob, y, activation="relu")
        torch.cuda.synchronize()
        sides.append((plan, blob, ws, x, h, y, y.clone(), h.clone(), torch.cuda.Stream()))
    for k in range(20):
        for plan, blob, ws, x, h, y, *_, stream in sides:
            plan.rms_norm_quantize(x, ws, residual=x, out=h, stream=stream)
            plan.matmul(ws, blob, y, activation="relu", stream=stream)
    torch.cuda.synchronize()
    for plan, blob, ws, x, h, y, want_y, want_h, _ in sides:
        assert torch.equal(y, want_y) and torch.equal(h, want_h)


def test_rows_up_to_the_plans(wq):
    """One plan, one workspace and one blob for every number of rows; y beyond the call's rows stays."""
    rng = np.random.default_rng(5)
    Cin, Cout, g, R = 512, 192, 64, 300
    plan, blob, ws, (wcodes, wscales), b = layer(wq, rng, R, Cin, Cout, g, 8)
    x = hidden(rng, R, Cin, "bf16")
    codes, scales = oracle.quantize_pixels(f32(x), g)
    z, S = lb.product(codes, scales, wcodes, wscales, b, g)
    xd = x.cuda()
    for n in (0, 1, 2, 15, 16, 17, 31, 32, 33, 48, 64, 65, 127, 128, 129, 255, 256, 300):
        print(n, flush=True)
        y = torch.full((R, Cout), float("nan"), dtype=torch.bfloat16, device="cuda")
        plan.linear(xd[:n], blob, ws, y[:n], activation="silu")
        torch.cuda.synchronize()
        check_product(y[:n], z[:n], S[:n], Cin // g, "silu", False, None)
        assert bool(y[n:].isnan().all())


def test_block_of_the_three(wq):
    """norm -> gated product -> product with residual, as a feed-forward block runs them, on a stream of its own, then from a
    captured graph replayed between eager passes: every pass has the same outputs, bit for bit."""
    rng = np.random.default_rng(9)
    for n, C, F, g, bits, dtype in ((1, 512, 1024, 64, 4, "bf16"), (45, 256, 704, 32, 8, "fp16"), (300, 512, 768, 128, 4, "fp32")):
        print(n, C, F, g, bits, dtype, flush=True)
        up, up_blob, up_ws, (uq, us), ub = layer(wq, rng, n, C, 2 * F, g, bits)
        down, down_blob, down_ws, (dq, ds), db = layer(wq, rng, n, F, C, g, bits)
        x, res = hidden(rng, n, C, dtype), hidden(rng, n, C, dtype)
        gamma = (1.0 + 0.2 * rng.standard_normal(C)).astype(np.float32)
        xd, rd, gd = x.cuda(), res.cuda(), torch.from_numpy(gamma).cuda()
        h, y = torch.empty_like(xd), torch.empty_like(xd)
        mid = xd.new_empty((n, F))
        torch.cuda.synchronize()

        def block():
            up.rms_norm_quantize(xd, up_ws, residual=rd, gamma=gd, out=h)
            up.matmul(up_ws, up_blob, mid, activation="silu", gated=True)
            down.linear(mid, down_blob, down_ws, y, residual=h)

        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            block()
        side.synchronize()
        hs, codes, scales = lb.rms_norm_quantize(f32(x), f32(res), gamma, 1e-6, g)
        assert torch.equal(h.cpu(), torch.from_numpy(hs).to(x.dtype))
        z, S = lb.product(codes, scales, uq, us, ub, g)
        check_product(mid, z, S, C // g, "silu", True, None)
        z, S = lb.product(*oracle.quantize_pixels(f32(mid), g), dq, ds, db, g)   # from the layer's own input
        check_product(y, z, S, F // g, "none", False, f32(h))

        want = (h.clone(), mid.clone(), y.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            block()
        for k in range(4):
            for t in (h, mid, y):
                t.zero_()
            graph.replay() if k % 2 == 0 else block()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, (h, mid, y))), k


def test_binding_refusals(wq):
    plan = wq.LinearPlan(4, 64, 64, 32)
    ws, blob = plan.alloc_workspace(), plan.alloc_blob()
    x, y = torch.zeros(4, 64, device="cuda"), torch.zeros(4, 64, device="cuda")
    plan.weight_prepare(torch.zeros(64, 64, device="cuda"), None, blob)
    with pytest.raises(TypeError):
        plan.quantize_rows(x.double(), ws)
    with pytest.raises(ValueError):
        plan.quantize_rows(x.t().contiguous().t(), ws)            # rows adjacent, not columns
    with pytest.raises(ValueError):
        plan.quantize_rows(torch.zeros(5, 64, device="cuda"), ws)
    with pytest.raises(ValueError):
        plan.quantize_rows(x.view(-1), ws)
    with pytest.raises(TypeError):
        plan.linear(x, blob, ws, y.half())
    with pytest.raises(ValueError):
        plan.linear(x, blob, ws, y, gated=True)
    with pytest.raises(ValueError):
        plan.linear(x, blob, ws, y, residual=y[:3])
    with pytest.raises(TypeError):
        plan.rms_norm_quantize(x, ws, gamma=torch.ones(64, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(wq.WqError):
        plan.linear(x, blob, ws[:16], y)
    with pytest.raises(wq.WqError):
        plan.rms_norm_quantize(x, ws, eps=0.0)
    with pytest.raises(wq.WqError):
        plan.linear(x[:1].expand(4, 64), blob, ws, y)            # one row four times: rows may not overlap
    plan.linear(x[:0], blob, ws, y[:0], residual=y[:0])
    plan.rms_norm_quantize(x[:0], ws, residual=x[:0], out=x[:0])
    plan.matmul(ws, blob, y[:0])

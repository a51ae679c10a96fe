"""Every tile of the 8-bit linear layer's products, in every way that they are formed, at sizes that the rules give to it.  What the codes stand
for comes from the library's own views (tested bit for bit elsewhere), the products from 64 bits on the GPU."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TILES = {"t256": 0, "t128": 1, "t128x64": 2, "t64": 3, "t64two": 4, "t64four": 5, "t64ring": 6, "t128two": 7}
# rows, Cin, Cout, gated
FORWARD = {
    "t256": (4090, 2100, 4090, False), "t256-gated": (4090, 2048, 8128, True),
    "t128": (1020, 2050, 8180, False), "t128-gated": (1020, 2048, 8128, True),
    "t128x64": (1000, 2310, 4600, False), "t128x64-gated": (1000, 2304, 4608, True),
    "t64": (1000, 700, 2555, False), "t64-gated": (1000, 640, 2560, True),
    "t64two": (1300, 1100, 1010, False), "t64two-gated": (1300, 1150, 1024, True),
    "t64four": (200, 2100, 500, False), "t64four-gated": (200, 2050, 448, True),
    "t64ring": (200, 900, 500, False), "t64ring-gated": (300, 1152, 1024, True),
    "t128two": (1000, 2100, 3450, False), "t128two-gated": (1000, 2050, 3456, True),
}
# rows, Cin, Cout: the gradient of x
INPUT_GRADS = {
    "t256": (4090, 4090, 2100), "t128": (1020, 8180, 2050), "t128x64": (1000, 4600, 1400), "t128two": (1000, 3450, 5130), "t64": (1000, 2555, 640),
    "t64two": (1100, 1250, 1100), "t64ring": (300, 1010, 1000),
}
# the gradient of the weights
WEIGHT_GRADS = {
    "t256": (1000, 4090, 4090), "t128": (1200, 2040, 4090), "t128x64": (300, 1280, 2870), "t64": (200, 1000, 2555),
    "t64two": (600, 1060, 1090), "t64ring": (1700, 500, 630),
}
# few rows: rows, Cin, Cout, gated
FEW = [
    (1, 4096, 640, False), (1, 8200, 640, True), (4, 2048, 4096, False), (7, 1000, 2048, True), (16, 640, 640, False), (16, 768, 10240, True),
    (16, 1152, 512, False), (16, 1152, 1024, True), (40, 500, 2000, False), (64, 300, 2304, True), (128, 640, 1760, False), (100, 640, 3584, True),
]


def quantized(v, dim):
    """What the codes of fp32 v with a scale for each 128 along dim stand for, in 64 bits."""
    if dim == 0:
        return quantized(v.t(), 1).t()
    R, C = v.shape
    p = torch.nn.functional.pad(v, (0, -C % 128)).view(R, -1, 128)
    m, e = torch.frexp(p.abs().amax(2))
    e = torch.where(p.abs().amax(2) > 0, e - 9 + (m > 0.875).int(), -126).clamp(-126, 127)
    s, r = ((e + 127) << 23).view(torch.float32), ((127 - e) << 23).view(torch.float32)
    return ((p * r[..., None]).to(torch.float8_e4m3fn).double() * s.double()[..., None]).view(R, -1)[:, :C]


def weights(wq, gen, rows, C, O, loaded, backward):
    plan = wq.Fp8LinearPlan(rows, C, O, backward=backward, fp32_scales=loaded)
    blob, ws = plan.alloc_blob(), plan.alloc_workspace()
    blob.fill_(0xFF)
    ws.fill_(0xFF)
    w = torch.randn((O, C), generator=gen, device="cuda") * 0.05
    bias = torch.randn((O,), generator=gen, device="cuda")
    if loaded:
        scales = torch.rand((math.ceil(O / 128), math.ceil(C / 128)), generator=gen, device="cuda") + 0.3
        plan.weight_load((w * 100).to(torch.float8_e4m3fn), scales * 1e-3, bias, blob)
    else:
        plan.weight_prepare(w, bias, blob)
    codes, scales, _ = plan.blob_views(blob)
    wide = scales.double().repeat_interleave(128, 0)[:O].repeat_interleave(128, 1)[:, :C]
    return plan, blob, ws, codes.double() * wide, bias.double()


def rows_of(gen, R, C, size=1.0):
    x = torch.randn((R, C), generator=gen, device="cuda") * torch.exp(0.5 * torch.randn((R, 1), generator=gen, device="cuda")) * size
    x[:, C // 3] *= 20.0
    x[R // 2] = 0.0
    return x


def check(got, want, S, K, direct):
    """A rounding of the magnitudes' sum for each of K terms; where codes are multiplied directly, up to seven of eight products are cut off at
    2^-13 of the largest; and the type's own rounding."""
    half = torch.finfo(got.dtype).eps / 2
    e = ((K + 16) * U + (7 * 2.0 ** -13 if direct else 0.0)) * S
    bad = ~((got.double() - want).abs() <= e * 1.01 + half * (want.abs() + e) + torch.finfo(got.dtype).smallest_normal * half)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:5].tolist())
    rms = ((got.double() - want).norm() / want.norm()).item()
    # roundings of either sign add up like their root; the direct products' cut is 1.5e-5 for values of like size, more where some are loud
    assert rms <= (4 + math.sqrt(K / 8)) * U + 0.6 * half * 2 + (2e-4 if direct else 0.0), rms


@pytest.mark.parametrize("loaded", [False, True], ids=["pow2", "any"])
@pytest.mark.parametrize("name", FORWARD)
def test_forward(wq, name, loaded):
    rows, C, O, gated = FORWARD[name]
    print(name, loaded, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + C + O)
    plan, blob, ws, w, bias = weights(wq, gen, rows, C, O, loaded, False)
    outs = O // 2 if gated else O
    for dtype in (torch.float32, torch.bfloat16):
        x = rows_of(gen, rows, C).to(dtype)
        X = quantized(x.float(), 1)
        z, S = X @ w.t() + bias, X.abs() @ w.abs().t() + bias.abs()
        y, pre = torch.full((rows, outs), float("nan"), device="cuda", dtype=dtype), torch.full((rows, O), float("nan"), device="cuda", dtype=dtype)
        plan.linear(x, blob, ws, y, gated=gated, preactivation=pre)
        check(pre, z, S, C, False)
        if gated:   # a product of two sums
            g, u = z[:, :outs], z[:, outs:]
            E = g.abs() * S[:, outs:] + u.abs() * S[:, :outs] + (C + 16) * U * S[:, outs:] * S[:, :outs]
            check(y, g * u, E, C, False)
        else:
            assert torch.equal(y, pre)


@pytest.mark.parametrize("loaded", [False, True], ids=["pow2", "any"])
@pytest.mark.parametrize("name", INPUT_GRADS)
def test_input_gradient(wq, name, loaded):
    rows, C, O = INPUT_GRADS[name]
    print(name, loaded, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + C + O)
    plan, blob, ws, w, _ = weights(wq, gen, rows, C, O, loaded, True)
    for dtype in (torch.float32, torch.bfloat16):
        dy = rows_of(gen, rows, O, 1e-2).to(dtype)
        D = quantized(dy.float(), 1)
        dx = torch.full((rows, C), float("nan"), device="cuda", dtype=dtype)
        plan.backward(None, dy, blob, ws, dx=dx)
        check(dx, D @ w, D.abs() @ w.abs(), O, dtype != torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("name", WEIGHT_GRADS)
def test_weight_gradient(wq, name, dtype):
    rows, C, O = WEIGHT_GRADS[name]
    print(name, dtype, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + C + O)
    plan = wq.Fp8LinearPlan(rows, C, O, backward=True)
    ws = plan.alloc_workspace()
    ws.fill_(0xFF)
    x, dy = rows_of(gen, rows, C).bfloat16(), rows_of(gen, rows, O, 1e-2).bfloat16()
    X, D = quantized(x.float(), 0), quantized(dy.float(), 0)
    dw = torch.full((O, C), float("nan"), device="cuda", dtype=dtype)
    db = torch.empty((O,), device="cuda")
    plan.backward(x, dy, None, ws, dw=dw, db=db)
    want, S = D.t() @ X, D.abs().t() @ X.abs()
    check(dw, want, S, rows, dtype != torch.float32)
    total = dy.double().abs().sum(0)
    assert bool(((db.double() - dy.double().sum(0)).abs() <= (rows + 4) * U * total).all())
    plan.backward(x, dy, None, ws, dw=dw, accumulate=True)
    half = torch.finfo(dtype).eps / 2
    check(dw, 2 * want, 2 * S + 2 * half / ((rows + 16) * U) * want.abs(), rows, dtype != torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("case", FEW, ids=lambda c: "%dx%d-%d%s" % (*c[:3], "-gated" if c[3] else ""))
def test_few_rows(wq, case, dtype):
    """One launch or two, in a stream or in a graph: the same bits.  The graph's input changes between its replays."""
    rows, C, O, gated = case
    print(case, dtype, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + C + O)
    plan, blob, ws, w, bias = weights(wq, gen, rows + 3, C, O, rows % 2 == 0, False)
    outs = O // 2 if gated else O
    xs = [rows_of(gen, rows, C).to(dtype) for _ in range(2)]
    want, y = [], torch.empty((rows, outs), device="cuda", dtype=dtype)
    for x in xs:
        plan.linear(x, blob, ws, y, gated=gated, activation="silu")
        want.append(y.clone())
        plan.quantize_rows(x, ws)
        y.fill_(float("nan"))
        plan.matmul(ws, blob, y, gated=gated, activation="silu")
        assert torch.equal(y, want[-1])
    X = quantized(xs[0].float(), 1)
    if not gated:
        got = torch.empty_like(y)
        plan.linear(xs[0], blob, ws, got)
        check(got, X @ w.t() + bias, X.abs() @ w.abs().t() + bias.abs(), C, False)
    x, own = xs[0].clone(), plan.alloc_workspace()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.linear(x, blob, own, y, gated=gated, activation="silu")
    for k in (0, 1, 1, 0):
        x.copy_(xs[k])
        y.fill_(float("nan"))
        graph.replay()
        assert torch.equal(y, want[k])
        plan.quantize_rows(xs[1 - k], ws)


@pytest.mark.parametrize("rows", [1, 16, 48, 300])
def test_results_over_the_input(wq, rows):
    """y may be x: the rows are quantized before the product writes any."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    plan, blob, ws, w, bias = weights(wq, gen, rows, 640, 640, False, True)
    x = rows_of(gen, rows, 640).bfloat16()
    want, pre = torch.empty_like(x), torch.empty_like(x)
    plan.linear(x, blob, ws, want, activation="gelu", residual=x, preactivation=pre)
    y = x.clone()
    plan.linear(y, blob, ws, y, activation="gelu", residual=y)
    assert torch.equal(y, want)
    y, z = x.clone(), x.clone()
    plan.linear(z, blob, ws, y, activation="gelu", residual=x, preactivation=z)
    assert torch.equal(y, want) and torch.equal(z, pre)
    # gradients over what they are of
    dy = rows_of(gen, rows, 640).bfloat16()
    dx, dw = torch.empty_like(x), torch.empty((640, 640), device="cuda")
    plan.backward(x, dy, blob, ws, dx=dx, dw=dw, preactivation=pre, activation="gelu")
    for over in range(3):
        t, dw2 = [x.clone(), dy.clone(), pre.clone()], torch.empty_like(dw)
        plan.backward(t[0], t[1], blob, ws, dx=t[over], dw=dw2, preactivation=t[2], activation="gelu")
        assert torch.equal(t[over], dx) and torch.equal(dw2, dw)


def test_two_graphs_share_a_workspace_in_order(wq):
    """Two captured steps, one after the other on a stream, may use one workspace: each call writes what it reads."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    plan, blob, ws, _, _ = weights(wq, gen, 200, 500, 384, False, True)
    sets = [(rows_of(gen, n, 500).bfloat16(), rows_of(gen, n, 384).bfloat16()) for n in (200, 130)]
    outs, want, graphs = [], [], []
    for x, dy in sets:
        o = [torch.empty_like(dy), torch.empty_like(x), torch.empty((384, 500), device="cuda"), torch.empty((384,), device="cuda")]
        step = lambda x=x, dy=dy, o=o: (plan.linear(x, blob, ws, o[0]), plan.backward(x, dy, blob, ws, dx=o[1], dw=o[2], db=o[3]))   # noqa: E731
        step()
        want.append([t.clone() for t in o])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        outs.append(o)
        graphs.append(graph)
    for k in (0, 1, 1, 0, 1):
        for t in outs[k]:
            t.fill_(float("nan"))
        ws.fill_(0xFF)
        graphs[k].replay()
        assert all(torch.equal(a, b) for a, b in zip(outs[k], want[k]))


def test_calls_of_other_numbers_of_rows(wq):
    """Calls of fewer rows leave the others' codes, and a product of fewer rows than were quantized has the same bits."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    for rows in (24, 200, 1000):
        plan, blob, ws, w, bias = weights(wq, gen, rows, 500, 384, False, False)
        x = rows_of(gen, rows, 500).half()
        y = torch.empty((rows, 384), device="cuda", dtype=x.dtype)
        plan.linear(x, blob, ws, y)
        plan.quantize_rows(x, ws)
        plan.quantize_rows(x[:7], ws)
        again = torch.full_like(y, float("nan"))
        plan.matmul(ws, blob, again)
        assert torch.equal(again, y)
        part = torch.full_like(y, float("nan"))
        plan.matmul(ws, blob, part[:rows - 5])
        assert bool(part[rows - 5:].isnan().all())
        X = quantized(x[:rows - 5].float(), 1)
        check(part[:rows - 5], X @ w.t() + bias, X.abs() @ w.abs().t() + bias.abs(), 500, False)


def test_a_nan_scale_makes_its_block_nan(wq):
    """e8m0 byte 255, in a plan of either kind, forward and backward; the other blocks' columns are what they were."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    codes = torch.randn((300, 200), generator=gen, device="cuda").to(torch.float8_e4m3fn)
    e = torch.full((3, 2), 127, dtype=torch.uint8, device="cuda")
    x, dy = rows_of(gen, 5, 200).bfloat16(), rows_of(gen, 5, 300).bfloat16()
    for any_scales in (False, True):
        plan = wq.Fp8LinearPlan(5, 200, 300, backward=True, fp32_scales=any_scales)
        blob, ws = plan.alloc_blob(), plan.alloc_workspace()
        got = []
        for byte in (127, 255):
            e[1, 0] = byte
            plan.weight_load(codes, e.view(torch.float8_e8m0fnu), None, blob)
            y, dx = torch.empty((5, 300), device="cuda", dtype=x.dtype), torch.empty_like(x)
            plan.linear(x, blob, ws, y)
            plan.backward(None, dy, blob, ws, dx=dx)
            got.append((y, dx))
        (y, dx), (yn, dxn) = got
        assert bool(yn[:, 128:256].isnan().all()) and torch.equal(yn[:, :128], y[:, :128]) and torch.equal(yn[:, 256:], y[:, 256:])
        assert bool(dxn[:, :128].isnan().all()) and torch.equal(dxn[:, 128:], dx[:, 128:])

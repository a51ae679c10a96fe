"""Kernel instances of the linear layer's surroundings that sizes alone choose, each at sizes inside the rule that chooses it
(tests/test_linear_forms.py checks on the CPU that these sizes do, and that no instance is left out)."""
import numpy as np
import pytest
import torch

import oracle
from oracle import linear_block as lb
from test_linear_block_gpu import NAMES, check_codes, check_product, f32, hidden, layer, rows_of

pytestmark = pytest.mark.gpu

# rows, weight rows (gated, not gated), Cin by group size, and what linear() and matmul() launch
SHORT = {32: 224, 64: 192, 128: 384, 256: 768, 512: 1024}
PRODUCTS = {
    "one launch": (13, (96, 93), SHORT, "rows1 x8 itself, rows1 x4"),
    "one launch, several blocks of rows": (35, (128, 125), SHORT, "rows1 x8 itself, rows1 x4"),
    "one launch, many columns": (3, (16416, 8203), SHORT, "rows1 x4 itself, rows1 x4"),
    "two launches": (16, (160, 75), {32: 1056, 64: 1088, 128: 1152, 256: 1280, 512: 1536}, "rows1 x4, rows1 x4"),
    "two blocks of rows": (101, (1280, 637), SHORT, "rows2 x4, rows2 x4"),
    "two blocks of rows, the second past the end": (17, (8256, 4125), SHORT, "rows2 x4, rows2 x4"),
}


@pytest.mark.parametrize("bits", [8, 4], ids=["w8", "w4"])
@pytest.mark.parametrize("g", SHORT)
@pytest.mark.parametrize("case", PRODUCTS)
def test_product_of_few_rows(wq, case, g, bits):
    """linear(), then matmul() of the codes that quantize_rows leaves, gated and not, every row and column."""
    n, couts, cins, _ = PRODUCTS[case]
    Cin = cins[g]
    for gated, Cout in zip((True, False), couts):
        print(case, g, bits, gated, flush=True)
        rng = np.random.default_rng(g + bits + n)
        plan, blob, ws, (wcodes, wscales), b = layer(wq, rng, n, Cin, Cout, g, bits)
        outs = Cout // 2 if gated else Cout
        x = hidden(rng, n, Cin, "bf16")
        res = torch.from_numpy(rng.standard_normal((n, outs)).astype(np.float32)).bfloat16()
        z, S = lb.product(*oracle.quantize_pixels(f32(x), g), wcodes, wscales, b, g)
        for call in ("linear", "matmul"):
            y = torch.full((n, outs), float("nan"), dtype=torch.bfloat16, device="cuda")
            if call == "linear":
                plan.linear(x.cuda(), blob, ws, y, activation="silu", gated=gated, residual=res.cuda())
            else:
                plan.quantize_rows(x.cuda(), ws)
                plan.matmul(ws, blob, y, activation="silu", gated=gated, residual=res.cuda())
            torch.cuda.synchronize()
            check_product(y, z, S, Cin // g, "silu", gated, f32(res))


@pytest.mark.parametrize("bits", [8, 4], ids=["w8", "w4"])
@pytest.mark.parametrize("g", SHORT)
def test_one_launch_has_the_bits_of_two(wq, g, bits):
    """linear() adds a column's groups in the order of matmul(), whichever quantizes the rows."""
    for n, Cin, Cout in ((1, 4 * SHORT[g], 544), (3, SHORT[g], 8224), (9, SHORT[g], 96), (16, 1024, 64), (40, SHORT[g], 160), (2, 4096, 96),
                         (90, SHORT[g], 1920), (300, SHORT[g], 4480)):
        print(n, Cin, Cout, g, bits, flush=True)
        plan, blob, ws, _, _ = layer(wq, np.random.default_rng(n), n, Cin, Cout, g, bits)
        x = hidden(np.random.default_rng(Cin), n, Cin, "fp32").cuda()
        for gated in (False, True):
            y = [torch.full((n, Cout // 2 if gated else Cout), float("nan"), device="cuda") for _ in range(2)]
            plan.linear(x, blob, ws, y[0], activation="gelu", gated=gated)
            plan.quantize_rows(x, ws)
            plan.matmul(ws, blob, y[1], activation="gelu", gated=gated)
            assert bool(y[0].isfinite().all()) and torch.equal(*y), (n, Cin, Cout, gated)


def test_captured_calls_of_both_forms(wq):
    """A graph of calls on either side of its own limit for one launch, replayed between eager passes: the same bits."""
    calls = []
    for n, Cin, Cout, g, bits in ((4, 4096, 256, 128, 4), (24, 1024, 96, 64, 8), (3, 4096, 96, 128, 8), (1, 16384, 64, 512, 4), (1, 12320, 64, 32, 8)):
        print(n, Cin, Cout, g, bits, flush=True)
        plan, blob, ws, _, _ = layer(wq, np.random.default_rng(n), n, Cin, Cout, g, bits)
        x = hidden(np.random.default_rng(Cin), n, Cin, "bf16").cuda()
        calls.append((plan, x, blob, ws, torch.empty((n, Cout), dtype=torch.bfloat16, device="cuda")))

    def run():
        for plan, x, blob, ws, y in calls:
            plan.linear(x, blob, ws, y, activation="silu", residual=None)

    run()
    torch.cuda.synchronize()
    want = [c[4].clone() for c in calls]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for k in range(5):
        for c in calls:
            c[4].fill_(float("nan"))
        graph.replay() if k % 2 == 0 else run()
        torch.cuda.synchronize()
        assert all(torch.equal(c[4], w) for c, w in zip(calls, want)), k


# rows, rows of the plan, Cin, g: two rows a wave, an odd number of rows and of a chunk's elements among them
MANY = [(1367, 1400, 1312, 32), (4096, 4097, 480, 32), (2049, 2050, 1088, 64), (4097, 4100, 512, 512), (2051, 2051, 896, 128),
        (1025, 1030, 1792, 256), (257, 300, 8192, 64), (4098, 4098, 32, 32)]


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("case", MANY, ids=lambda c: "%dof%d_%d_g%d" % c)
def test_codes_of_many_rows(wq, case, dtype):
    """Bit for bit, with the rows behind the last one left as they were."""
    n, R, C, g = case
    print(case, dtype, flush=True)
    rng = np.random.default_rng(n + C)
    plan = wq.LinearPlan(R, C, 32, g)
    x = hidden(rng, n, C, dtype)
    x[n - 1, ::3] = 5.0
    codes, scales = oracle.quantize_pixels(f32(x), g)
    for pad, off in ((0, 0), (16, 16)):
        ws = plan.alloc_workspace()
        ws.fill_(0xA5)
        before = [v[n:].cpu().numpy().tobytes() for v in plan.workspace_views(ws)]
        plan.quantize_rows(rows_of(x, C + pad, off), ws)
        torch.cuda.synchronize()
        check_codes(plan, ws, n, codes, scales)
        assert before == [v[n:].cpu().numpy().tobytes() for v in plan.workspace_views(ws)]


# rows, rows of the plan, Cin, g: rows of more than 16384 elements, eight pieces a lane
WIDE = [(3, 5, 16896, 64), (2, 2, 32768, 512), (3, 3, 16416, 32), (5, 9, 16512, 128), (1, 1, 24576, 256)]


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("case", WIDE, ids=lambda c: "%dof%d_%d_g%d" % c)
def test_norm_of_wide_rows(wq, case, dtype):
    n, R, C, g = case
    print(case, dtype, flush=True)
    rng = np.random.default_rng(n + C)
    plan = wq.LinearPlan(R, C, 32, g)
    x, res = hidden(rng, n, C, dtype), hidden(rng, n, C, dtype)
    gamma = (1.0 + 0.2 * rng.standard_normal(C)).astype(np.float32)
    for with_res, with_gamma in ((True, True), (False, False), (True, False)):
        ws = plan.alloc_workspace()
        ws.fill_(0xA5)
        before = [v[n:].cpu().numpy().tobytes() for v in plan.workspace_views(ws)]
        xd, rd = rows_of(x, C + 8, 8), rows_of(res, C + 8, 8) if with_res else None
        h = torch.empty_like(xd)
        plan.rms_norm_quantize(xd, ws, residual=rd, gamma=torch.from_numpy(gamma).cuda() if with_gamma else None, eps=1e-5, out=h)
        torch.cuda.synchronize()
        hs, codes, scales = lb.rms_norm_quantize(f32(x), f32(res) if with_res else None, gamma if with_gamma else None, 1e-5, g)
        check_codes(plan, ws, n, codes, scales)
        assert torch.equal(h.cpu(), torch.from_numpy(hs).to(x.dtype))
        assert before == [v[n:].cpu().numpy().tobytes() for v in plan.workspace_views(ws)]

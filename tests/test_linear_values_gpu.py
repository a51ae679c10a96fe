"""Values at which the linear layer's surroundings can go wrong: infinities and NaN, activations by place, the norm's factor
next to a rounding's border, sums over many groups."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import linear_block as lb

pytestmark = pytest.mark.gpu

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
ROWS = {"rows": 1, "tiles": 130}   # the two kernels' epilogues


def through(wq, z, act, n, gated=False):
    """act(z) [n][len(z)] in fp32, as a layer's epilogue computes it: rows of zeros, so that the products are the bias."""
    C = z.numel()
    assert C % 4096 == 0   # enough columns for the tiled kernels at 130 rows
    bias = torch.cat((z, torch.ones(C))) if gated else z
    plan = wq.LinearPlan(n, 32, bias.numel(), 32)
    blob, ws = plan.alloc_blob(), plan.alloc_workspace()
    plan.weight_prepare(torch.ones(bias.numel(), 32, device="cuda"), bias.cuda(), blob)
    y = torch.full((n, C), 7.0, device="cuda")
    plan.linear(torch.zeros(n, 32, device="cuda"), blob, ws, y, activation=act, gated=gated)
    return y.cpu()


def exact(z, act):
    """The activation's formula in 64 bits; gelu by erfc, which keeps the negative tail's digits."""
    z = z.double()
    if act == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), z)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return z * torch.erfc(z * -math.sqrt(0.5)) * 0.5
    if act == "gelu_tanh":
        return z / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("act", ACTS)
def test_activations_of_infinities_and_nan(wq, act, rows, gated):
    """What the formulas give: NaN stays NaN, +inf stays +inf, -inf is -inf, 0 (relu) or the undefined -inf times 0."""
    print(act, rows, gated, flush=True)
    special = torch.tensor([math.nan, math.inf, -math.inf, 3e38, -3e38, 0.0, -0.0, 1e30, -1e30, 1e-30])
    z = torch.zeros(4096)
    z[5:4085].view(-1, 10)[:, :] = special
    y = through(wq, z, act, ROWS[rows], gated)
    want = exact(z, act).float()
    for r in range(y.shape[0]):
        assert torch.equal(y[r].isnan(), want.isnan())
        assert torch.equal(y[r].nan_to_num(1.0, 2e38, -2e38).abs() > 1e37, want.nan_to_num(1.0, 2e38, -2e38).abs() > 1e37)
        assert torch.equal(y[r].isinf(), want.isinf()) and torch.equal(y[r] > 0, want > 0)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("act", ACTS)
def test_activations_by_place(wq, act, rows):
    """The error of each value against itself, not against the largest: what include/wq.h states, from counted roundings.  u = 2^-24.
      silu: the exponent's argument is off by 1.22 u of itself (its constant by 0.22), the exponential and the reciprocal by a unit
        in the last place (2 u) each, the sum and the product by u: 6 u + 1.22 u |z|;
      gelu_tanh: a square, a multiply-add and a product form the argument, their constants are off by 0.33 u: 3.4 u of it;
      gelu: z^2 / 2 is off by 2.3 u of itself, the polynomial by 15 u at most down to -8 and by 21 u to -10 (its rounding steps, the
        reciprocal's error in its argument, and 1.2 u to -6, 8 u to -8, 14 u to -10 of the fit), the exponential by 2 u, two products and the sum by u each;
      the hardware flushes reciprocals below 2^-126, so that z times one is off by 2^-118 at most (|z| < 256)."""
    print(act, rows, flush=True)
    z = torch.cat((torch.linspace(-14, 14, 40000), torch.linspace(-120, -14, 8000), torch.linspace(14, 200, 1536),
                   torch.logspace(-36, 0, 8000), -torch.logspace(-36, 0, 8000)))
    y = through(wq, z, act, ROWS[rows])
    want, wide, u = exact(z, act), z.double(), 2.0 ** -24
    arg = 2.0 * math.sqrt(2.0 / math.pi) * (wide.abs() + 0.044715 * wide.abs() ** 3)
    steps = {"none": 0.0 * wide, "relu": 0.0 * wide, "silu": 8.0 + 1.3 * wide.abs(), "gelu": 24.0 + 2.0 * wide ** 2,
             "gelu_tanh": 8.0 + 3.5 * arg}[act]
    bound = steps * u * want.abs() + (2.0 ** -118 if act in ("silu", "gelu_tanh") else 2.0 ** -149)
    if act == "gelu":
        bound = torch.where(wide < -10, 2.0 ** -80 * torch.ones_like(wide), bound)
    for r in (0, y.shape[0] - 1):
        off = (y[r].double() - want).abs()
        worst = int((off / bound).argmax())
        print("row %d: %.3f of the bound at %g" % (r, float(off[worst] / bound[worst]), float(z[worst])), flush=True)
        assert bool((off <= bound).all())


@pytest.mark.parametrize("g", [32, 64, 128, 256, 512])
def test_codes_of_infinities_and_nan(wq, g):
    """Rows with infinities and NaN have the codes and scales that the older quantizer gives them, wherever the rows lie: a group
    with a NaN a scale of zero, one with an infinity an infinite scale, and every other group its own."""
    print(g, flush=True)
    R, C = 6, 4 * g
    gen = torch.Generator().manual_seed(g)
    x = torch.randn(R, C, generator=gen)
    x[0, 3] = math.nan
    x[1, g + 5] = math.inf
    x[2, 2 * g + 1], x[2, 2 * g + 9] = -math.inf, math.nan
    x[3, C - 1] = -math.nan
    x[4] = math.nan
    plan = wq.LinearPlan(R, C, 32, g)
    ws = plan.alloc_workspace()
    plan.quantize(x.cuda(), ws)
    codes, scales = plan.workspace_views(ws)
    kept = scales.cpu()
    assert kept[0, 0] == 0 and kept[1, 1] == math.inf and kept[2, 2] == 0 and kept[3, 3] == 0 and not kept[4].any() and kept[5].all()
    for pad, off in ((0, 0), (16, 4), (3, 1)):
        v = torch.zeros(off + R * (C + pad), device="cuda")[off:].view(R, C + pad)[:, :C]
        v.copy_(x)
        ws.fill_(0xA5)
        plan.quantize_rows(v, ws)
        c, s = plan.workspace_views(ws)
        assert torch.equal(s.cpu(), kept), (pad, off)
        assert torch.equal(c, codes), (pad, off)


@pytest.mark.parametrize("act", ACTS)
def test_infinities_and_nan_stay_in_their_row(wq, act):
    """An infinity in a row of x makes that row of y NaN, through every activation, and leaves the others alone."""
    for n, Cin, Cout in ((3, 256, 64), (40, 2048, 64), (130, 256, 4096)):
        print(act, n, flush=True)
        gen = torch.Generator().manual_seed(n)
        plan = wq.LinearPlan(n, Cin, Cout, 64)
        blob, ws = plan.alloc_blob(), plan.alloc_workspace()
        plan.weight_prepare(torch.randn(Cout, Cin, generator=gen).cuda(), None, blob)
        x = torch.randn(n, Cin, generator=gen).cuda()
        want, y = torch.empty(n, Cout, device="cuda"), torch.empty(n, Cout, device="cuda")
        plan.linear(x, blob, ws, want, activation=act)
        x[1, 70] = math.inf
        plan.linear(x, blob, ws, y, activation=act)
        rest = [r for r in range(n) if r != 1]
        assert bool(y[1].isnan().all()) and torch.equal(y[rest], want[rest]) and bool(want.isfinite().all())


@pytest.mark.parametrize("C,g", [(4096, 128), (1280, 64), (512, 512), (32, 32), (13312, 256), (32768, 512)])
def test_the_norms_codes_do_not_depend_on_where_rows_lie(wq, C, g):
    """Rows in aligned pieces and rows at odd addresses go through different kernels.  Where the norm's factor lies next to the
    middle between two fp32 numbers, the last place of a sum of squares decides it: eps is moved over such a place in the smallest
    steps of 64 bits, and all codes and scales stay alike."""
    plan = wq.LinearPlan(1, C, 32, g)
    even, odd = plan.alloc_workspace(), plan.alloc_workspace()
    even.zero_(), odd.zero_()   # (what lies between codes and scales is compared too)
    moved = 0
    for seed in range(12):
        print(C, g, seed, flush=True)
        x = np.random.default_rng(seed).standard_normal(C).astype(np.float32)
        mean = math.fsum((x.astype(np.float64) ** 2).tolist()) / C
        low = np.float32(1.0 / math.sqrt(mean + 1e-3))
        middle = (float(low) + float(np.nextafter(low, np.float32(0)))) / 2.0   # factors round differently on its two sides
        eps = 1.0 / (middle * middle) - mean
        step = float(np.spacing(1.0 / (middle * middle)))
        a = torch.from_numpy(x).cuda().view(1, C)
        flat = torch.zeros(C + 1, device="cuda")
        flat[1:] = a[0]
        scales = set()
        for k in range(-16, 17):
            plan.rms_norm_quantize(a, even, eps=eps + k * step)
            plan.rms_norm_quantize(flat[1:].view(1, C), odd, eps=eps + k * step)
            same = torch.equal(even, odd)
            assert same, (seed, k)
            scales.add(float(plan.workspace_views(even)[1][0, 0]))
        moved += len(scales) == 2
    assert moved >= 6   # such places were met


# rows and weight rows of the forms that add all groups of a column one after the other, and of the others
LONG = {"rows": (5, 96), "rows2": (50, 1440), "teams4": (199, 2240), "teams2": (301, 4480), "teams1": (641, 4480), "large": (2501, 4480)}


@pytest.mark.parametrize("form", LONG)
def test_sums_over_many_groups(wq, form):
    """256 groups of 32 in fp32.  n terms of either sign, of size s, add up to some s sqrt(n); the k-th addition rounds a sum of
    s sqrt(k) by up to u of it, and independent roundings add up to u s sqrt(n (n + 1) / 2): sqrt((n + 1) / 2) u of the result
    where nothing splits the sum.  Each term's two products and the bias add less than 3 u.  Root mean squares over the sample."""
    n, Cout = LONG[form]
    print(form, flush=True)
    rng = np.random.default_rng(n)
    Cin, g, u = 8192, 32, 2.0 ** -24
    plan = wq.LinearPlan(n, Cin, Cout, g)
    blob, ws = plan.alloc_blob(), plan.alloc_workspace()
    gen = torch.Generator(device="cuda").manual_seed(n)
    w = torch.randn((Cout, Cin), generator=gen, device="cuda") * 0.05
    x = torch.randn((n, Cin), generator=gen, device="cuda")
    plan.weight_prepare(w, None, blob)
    y = torch.empty((n, Cout), device="cuda")
    plan.linear(x, blob, ws, y)
    rows, cols = sorted(set(rng.integers(0, n, 12).tolist())), sorted(set(rng.integers(0, Cout, 96).tolist()))
    wcodes, wscales = oracle.quantize_weight_rows(w[cols].cpu().numpy(), g, 8)
    z, _ = lb.product(*oracle.quantize_pixels(x[rows].cpu().numpy(), g), wcodes, wscales, None, g)
    e = y[rows][:, cols].double().cpu().numpy() - z
    rms = float(np.sqrt((e ** 2).mean() / (z ** 2).mean()))
    print("rms %.2e, %.2f u" % (rms, rms / u), flush=True)
    assert rms <= (math.sqrt((Cin // g + 1) / 2) + 3.0) * u

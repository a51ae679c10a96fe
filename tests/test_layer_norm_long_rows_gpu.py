"""Layer norm's gradient of rows of thousands to hundreds of millions of columns, against 64 bits on the GPU."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
NAMES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def inputs(n, C, dtype):
    gen = torch.Generator(device="cuda").manual_seed(n * 7 + C)
    h = torch.randn((n, C), generator=gen, device="cuda").add_(0.5)
    h[:, C // 3] *= 20.0
    dy = torch.randn((n, C), generator=gen, device="cuda").mul_(1e-2)
    dy[n // 2, ::2] = 0.0
    gamma = 1.0 + 0.2 * torch.randn((C,), generator=gen, device="cuda")
    return dy.to(dtype), h.to(dtype), gamma


def wanted(dy, h, gamma, eps):
    """(value, how far roundings may take it) of dx, dgamma, dbeta."""
    dy, h, C = dy.double(), h.double(), h.shape[1]
    n = h - h.mean(1, keepdim=True)
    r = 1 / torch.sqrt((n * n).mean(1, keepdim=True) + eps)
    n *= r
    g = dy * gamma.double()
    mg, mgn = g.mean(1, keepdim=True), (g * n).mean(1, keepdim=True)
    # The means are sums in 64 bits of g = fl(dy gamma), each off by up to U |g|.  They, n (two roundings), its product with the second mean,
    # two differences, r and the product with it are rounded to fp32.
    means = U * (g.abs().mean(1, keepdim=True) + n.abs() * (g * n).abs().mean(1, keepdim=True))
    ex = r * (10 * U * (g.abs() + mg.abs() + (n * mgn).abs()) + means)
    # rows one after the other in fp32, then 64 bits; n is off by two roundings
    rows = (h.shape[0] / 100 + 30) * U
    return (r * (g - mg - n * mgn), ex), ((dy * n).sum(0), rows * (dy * n).abs().sum(0)), (dy.sum(0), rows * dy.abs().sum(0))


def check(got, want, e):
    half = torch.finfo(got.dtype).eps / 2
    bad = ~((got.double() - want).abs() <= e * 1.01 + half * (want.abs() + e) + torch.finfo(got.dtype).smallest_normal * half)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:5].tolist())


def run(wq, n, C, dtype, over):
    """All gradients in one call, dx in a tensor of its own, over h or over dy; then the weight's and bias's added to what they are."""
    print(n, C, dtype, over, flush=True)
    norm = wq.LayerNormPlan(n, C)
    dy, h, gamma = inputs(n, C, dtype)
    wants = wanted(dy, h, gamma, 1e-5)
    ws = norm.alloc_workspace()
    ws.fill_(0xFF)
    dgamma, dbeta = torch.full((C,), float("nan"), device="cuda"), torch.full((C,), float("nan"), device="cuda")
    hd, dyd = h.clone(), dy.clone()
    dx = {"h": hd, "dy": dyd, None: torch.full_like(dy, float("nan"))}[over]
    norm.backward(dyd, hd, ws, dx=dx, gamma=gamma, eps=1e-5, dgamma=dgamma, dbeta=dbeta)
    for got, (want, e) in zip((dx, dgamma, dbeta), wants):
        check(got, want, e)
    norm.backward(dy, h, ws, gamma=gamma, eps=1e-5, dgamma=dgamma, dbeta=dbeta, accumulate=True)
    for got, (want, e) in zip((dgamma, dbeta), wants[1:]):
        check(got, 2 * want, 2 * e)


# A launch has up to 2^16 workgroups along the columns, 64 of them to a workgroup at a time: from 2^21 columns on (dgamma and dbeta together), and from
# 2^22 on for the partial sums, each takes more than one block.  At 2^27 a workgroup of 1024 for each block would be 2^32 lanes.
@pytest.mark.parametrize("n,C,over", [(3, (1 << 22) + (1 << 21) + 77, "h"), (70, (1 << 22) + 8, None), (1, (1 << 27) + 40, "h")])
def test_more_columns_than_a_launch_has_workgroups_for(wq, n, C, over):
    run(wq, n, C, torch.bfloat16, over)


def test_the_longest_row(wq):
    """2^30 columns, forward and backward; compared a piece at a time."""
    C, piece = 1 << 30, 1 << 27
    gen = torch.Generator(device="cuda").manual_seed(30)
    norm = wq.LayerNormPlan(1, C)
    h, dy = (torch.randn((1, C), generator=gen, device="cuda").bfloat16() for _ in range(2))
    h += 0.5
    total = lambda f: sum(float(f(h[0, i:i + piece].double(), dy[0, i:i + piece].double()).sum()) for i in range(0, C, piece))   # noqa: E731
    mean = total(lambda a, d: a) / C
    r = (total(lambda a, d: (a - mean) ** 2) / C + 1e-5) ** -0.5
    mg, mgn = total(lambda a, d: d) / C, total(lambda a, d: d * (a - mean)) * r / C
    y = torch.full_like(h, float("nan"))
    norm.forward(h, y)
    dgamma, dbeta, ws = torch.full((C,), float("nan"), device="cuda"), torch.full((C,), float("nan"), device="cuda"), norm.alloc_workspace()
    dx = dy.clone()
    norm.backward(dx, h, ws, dx=dx, dgamma=dgamma, dbeta=dbeta)
    for i in range(0, C, piece):
        s = slice(i, i + piece)
        n, d = (h[0, s].double() - mean) * r, dy[0, s].double()
        check(y[0, s], n, 8 * U * n.abs())
        check(dx[0, s], r * (d - mg - n * mgn), 10 * U * r * (d.abs() + abs(mg) + (n * mgn).abs()))
        check(dgamma[s], d * n, 30 * U * (d * n).abs())
        assert torch.equal(dbeta[s], dy[0, s].float())


# nine to sixteen waves to a row and several rows to each (8193 to 16384 columns); longer rows, whose columns are added up by 64 units of four waves
@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("n,C,over", [(600, 8200, "dy"), (520, 12001, None), (700, 16384, "h"), (70, 16392, None), (300, 16400, "h")])
def test_several_rows_to_each_wave(wq, n, C, over, dtype):
    run(wq, n, C, NAMES[dtype], over)

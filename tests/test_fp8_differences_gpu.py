"""Gradients of the 8-bit linear layer against differences of its own results, with bounds that are a small part of what is compared.

Inputs and weights move by whole steps of their codes along the sign of the gradient, so that the codes' scales stay, the difference of two
results is linear in the step, and every term of gradient x step has the same sign: a gradient that is wrong, negated, scaled or in another
column's place misses by some or all of what moved."""
import numpy as np
import pytest
import torch

from oracle import fp8_block as fb
from test_fp8_gpu import U, check, f64

pytestmark = pytest.mark.gpu

STEP = 4.0
# rows, Cin, Cout: few rows and tiles of three sizes
LAYERS = [(1, 256, 96), (40, 256, 128), (128, 384, 2000), (300, 640, 1100), (600, 1280, 2400)]


def whole(rng, shape):
    """Multiples of 4 from 16 to 28 in size, of either sign: e4m3 numbers, as are the next multiples of 4 on both sides."""
    return (rng.choice([16.0, 20.0, 24.0, 28.0], shape) * rng.choice([-1.0, 1.0], shape)).astype(np.float32)


def dev(v):
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).cuda()


def same(got, want, room, part):
    """got = want but for `room`, which is at most `part` of it."""
    assert (room <= part * np.abs(want)).all(), float((room / np.abs(want)).max())
    assert (np.abs(got - want) <= room).all(), float((np.abs(got - want) / room).max())


@pytest.mark.parametrize("loaded", [False, True], ids=["pow2", "any"])
@pytest.mark.parametrize("case", LAYERS, ids=lambda c: "%dx%d-%d" % c)
def test_gradient_of_x(wq, case, loaded):
    n, C, O = case
    print(case, loaded, flush=True)
    rng = np.random.default_rng(n + C + O)
    plan = wq.Fp8LinearPlan(n, C, O, backward=True, fp32_scales=loaded)
    blob, ws = plan.alloc_blob(), plan.alloc_workspace()
    if loaded:
        codes = dev(rng.standard_normal((O, C)) * 30).to(torch.float8_e4m3fn)
        plan.weight_load(codes, dev(rng.random((-(-O // 128), -(-C // 128))) * 1e-3 + 1e-3), None, blob)
    else:
        plan.weight_prepare(dev(rng.standard_normal((O, C)) * 0.05), None, blob)
    codes, scales, _ = plan.blob_views(blob)
    w = f64(codes.float()) * np.repeat(np.repeat(f64(scales), 128, 0)[:O], 128, 1)[:, :C]
    dy = rng.choice([-1.0, 0.5, 2.0], (n, O)).astype(np.float32)   # every one of them a code
    dx = torch.empty((n, C), device="cuda")
    plan.backward(None, dev(dy), blob, ws, dx=dx)
    lo = whole(rng, (n, C))
    step = (STEP * np.sign(f64(dx))).astype(np.float32)
    lo[:, ::128], step[:, ::128] = 448.0, 0.0   # every group's scale is 1
    ys = []
    for x in (lo, lo + step):
        y = torch.empty((n, O), device="cuda")
        plan.linear(dev(x), blob, ws, y)
        ys.append(f64(y))
    # sums of C products, a rounding of the magnitudes' sum for each, and the result's own rounding
    ey = [(C + 16) * U * (np.abs(x) @ np.abs(w).T) + U * np.abs(y) for x, y in zip((lo, lo + step), ys)]
    change = step.astype(np.float64) @ w.T
    assert (np.abs(ys[1] - ys[0] - change) <= ey[0] + ey[1]).all()
    # row by row: what the loss moves is the gradient's product with the step
    ex = (O + 16) * U * (np.abs(dy).astype(np.float64) @ np.abs(w)) + U * np.abs(f64(dx))
    room = (np.abs(dy) * (ey[0] + ey[1])).sum(1) + (np.abs(step) * ex).sum(1)
    same((dy * (ys[1] - ys[0])).sum(1), (f64(dx) * step).sum(1), room, 0.1)


@pytest.mark.parametrize("case", LAYERS[:4], ids=lambda c: "%dx%d-%d" % c)
def test_gradient_of_the_weights(wq, case):
    n, C, O = case
    print(case, flush=True)
    rng = np.random.default_rng(n + C + O + 1)
    plan = wq.Fp8LinearPlan(n, C, O, backward=True)
    blob, ws = plan.alloc_blob(), plan.alloc_workspace()
    x = whole(rng, (n, C))   # the same codes in groups along a row and down a column: their largest are 16 to 28
    dy = rng.choice([-1.0, 0.5, 2.0], (n, O)).astype(np.float32)
    dw, db = torch.empty((O, C), device="cuda"), torch.empty(O, device="cuda")
    plan.backward(dev(x), dev(dy), None, ws, dw=dw, db=db)
    assert np.array_equal(f64(db), dy.astype(np.float64).sum(0))   # multiples of a half
    lo = whole(rng, (O, C))
    step = (STEP * np.sign(f64(dw))).astype(np.float32)
    lo[::128, ::128], step[::128, ::128] = 448.0, 0.0   # every block's scale is 1
    ys = []
    for w in (lo, lo + step):
        plan.weight_prepare(dev(w), None, blob)
        y = torch.empty((n, O), device="cuda")
        plan.linear(dev(x), blob, ws, y)
        ys.append(f64(y))
    ey = [(C + 16) * U * (np.abs(x).astype(np.float64) @ np.abs(w).T) + U * np.abs(y) for w, y in zip((lo, lo + step), ys)]
    ew = (n + 16) * U * (np.abs(dy).astype(np.float64).T @ np.abs(x)) + U * np.abs(f64(dw))
    # weight row by weight row
    room = (np.abs(dy) * (ey[0] + ey[1])).sum(0) + (np.abs(step) * ew).sum(1)
    same((dy * (ys[1] - ys[0])).sum(0), (f64(dw) * step).sum(1), room, 0.1)


@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh"])
def test_gradient_through_the_epilogue(wq, act, gated):
    """The bias is in fp32 and is not quantized: its gradient, the sum of dz, against a small step of it up and down."""
    rng = np.random.default_rng(len(act))
    n, C, O = 30, 64, 256
    outs = O // 2 if gated else O
    plan = wq.Fp8LinearPlan(n, C, O, backward=True)
    blob, ws = plan.alloc_blob(), plan.alloc_workspace()
    w, b = rng.standard_normal((O, C)) * 0.1, rng.standard_normal(O)
    x, dy = dev(rng.standard_normal((n, C))), rng.random((n, outs)) + 0.5
    y, pre, db = torch.empty((n, outs), device="cuda"), torch.empty((n, O), device="cuda"), torch.empty(O, device="cuda")
    plan.weight_prepare(dev(w), dev(b), blob)
    plan.linear(x, blob, ws, y, activation=act, gated=gated, preactivation=pre)
    plan.backward(None, dev(dy), None, ws, db=db, preactivation=pre, activation=act, gated=gated)
    h = 2.0 ** -6
    d = np.sign(f64(db))
    ys = []
    for sign in (1.0, -1.0):
        plan.weight_prepare(dev(w), dev(b.astype(np.float32) + (sign * h * d).astype(np.float32)), blob)
        plan.linear(x, blob, ws, y, activation=act, gated=gated)
        ys.append(f64(y))
    z = f64(pre)
    dyd = f64(dev(dy))
    got, want = (dyd * (ys[0] - ys[1])).sum(0) / (2 * h), f64(db) * d
    if gated:
        want = want[:outs] + want[outs:]
    # a result is off by its sum's rounding through a slope of at most 1.13, by 16 units of the activation, and by the other half's; the bias
    # by its own; what is left out is the third derivative's share, step^2 / 6 of act''' (below 2) of each, with a gate also of 3 act'' (below 3.4)
    S = np.abs(f64(x)) @ np.abs(w).T * 1.2 + np.abs(b) + 1   # (codes are up to a sixteenth larger, on both sides)
    size = 1.0 + np.abs(z)
    one = (C + 16) * U * S * 1.13 + 16 * U * size
    third = h * h / 6 * 2.0 if act != "none" else 0.0
    if gated:
        g, u = slice(0, outs), slice(outs, O)
        e = one[:, g] * size[:, u] + one[:, u] * size[:, g]
        third = third * (size[:, u] + 1.7) if act != "none" else 0.0
    else:
        e = one
    room = (dyd * (e / h + third)).sum(0) + 2 * (n + 20) * U * (dyd * (size[:, :outs] * size[:, outs:] if gated else size)).sum(0)
    # of one column the steps' shares may nearly cancel: the columns are compared one by one, the size of the room over all of them
    assert (np.abs(got - want) <= room).all(), float((np.abs(got - want) / room).max())
    assert room.sum() <= 0.05 * np.abs(want).sum(), room.sum() / np.abs(want).sum()


# rows, Cin, Cout
@pytest.mark.parametrize("n,C,O", [(5, 300, 192), (200, 384, 704), (640, 500, 1088)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])
def test_a_gate_without_an_activation(wq, n, C, O, dtype):
    """dz is dy times the other half."""
    rng = np.random.default_rng(n + C)
    plan = wq.Fp8LinearPlan(n, C, O, backward=True)
    blob, ws = plan.alloc_blob(), plan.alloc_workspace()
    plan.weight_prepare(dev(rng.standard_normal((O, C)) * 0.05), None, blob)
    codes, scales, _ = plan.blob_views(blob)
    w = f64(codes.float()) * np.repeat(np.repeat(f64(scales), 128, 0)[:O], 128, 1)[:, :C]
    # few significant bits: a product of two of them is an fp32 number, and its codes are certain
    few = lambda shape, s: torch.from_numpy((rng.integers(-31, 32, shape) * s).astype(np.float32)).to(dtype)   # noqa: E731
    x, dy, pre = few((n, C), 0.125), few((n, O // 2), 2.0 ** -6), few((n, O), 0.125)
    z = f64(pre)
    dz = np.concatenate([f64(dy) * z[:, O // 2:], f64(dy) * z[:, :O // 2]], 1)
    D1, D2, X2 = fb.through(dz), fb.through(dz.T).T, fb.through(f64(x).T).T
    Sx, Sw = np.abs(D1) @ np.abs(w), np.abs(D2).T @ np.abs(X2)
    cut = 7 * 2.0 ** -13   # of eight products of codes up to seven are cut off at 2^-13 of the largest
    for wide in (False, True):
        T = torch.float32 if wide else dtype
        dx, dw, db = torch.empty((n, C), dtype=dtype, device="cuda"), torch.empty((O, C), dtype=T, device="cuda"), torch.empty(O, device="cuda")
        plan.backward(x.cuda(), dy.cuda(), blob, ws, dx=dx, dw=dw, db=db, preactivation=pre.cuda(), gated=True)
        check(dx, D1 @ w, ((O + 16) * U + (0 if dtype == torch.float32 else cut)) * Sx)
        check(dw, D2.T @ X2, ((n + 16) * U + (0 if T == torch.float32 else cut)) * Sw)
        check(db, dz.sum(0), (n + 4) * U * np.abs(dz).sum(0))

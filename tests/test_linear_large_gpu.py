"""The linear layer's surroundings at the ends of what they take: rows that lie further apart than 32 bits count, and as many rows as
a plan may have."""
import numpy as np
import pytest
import torch

import oracle
from oracle import linear_block as lb
from test_linear_block_gpu import check_codes, check_product, f32, hidden, layer

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("off", [0, 1], ids=["aligned", "odd"])
def test_rows_further_apart_than_32_bits(wq, off):
    """40 rows, 2^27 elements from each to the next: the last ones' offsets pass 2^32 elements."""
    n, Cin, g, stride = 40, 512, 64, (1 << 27) + 64
    rng = np.random.default_rng(off)
    x, gamma = hidden(rng, n, Cin, "bf16"), (1.0 + 0.2 * rng.standard_normal(Cin)).astype(np.float32)
    flat = torch.empty(2, n * stride + 8, dtype=torch.bfloat16, device="cuda")
    far = [f[off:off + n * stride].view(n, stride) for f in flat]
    xd, h = (f[:, :Cin] for f in far)
    xd.copy_(x)
    for Cout in (96, 8256):   # few columns: one launch; many: tiles
        print(off, Cout, flush=True)
        plan, blob, ws, (wcodes, wscales), b = layer(wq, rng, n, Cin, Cout, g, 8)
        codes, scales = oracle.quantize_pixels(f32(x), g)
        plan.quantize_rows(xd, ws)
        torch.cuda.synchronize()
        check_codes(plan, ws, n, codes, scales)
        y = far[1][:, Cin:Cin + Cout]
        res = torch.from_numpy(rng.standard_normal((n, Cout)).astype(np.float32)).bfloat16()
        y.copy_(res)
        plan.linear(xd, blob, ws, y, activation="silu", residual=y)
        torch.cuda.synchronize()
        z, S = lb.product(codes, scales, wcodes, wscales, b, g)
        check_product(y, z, S, Cin // g, "silu", False, f32(res))
        plan.rms_norm_quantize(xd, ws, residual=xd, gamma=torch.from_numpy(gamma).cuda(), out=h)
        torch.cuda.synchronize()
        hs, codes, scales = lb.rms_norm_quantize(f32(x), f32(x), gamma, 1e-6, g)
        check_codes(plan, ws, n, codes, scales)
        assert torch.equal(h.cpu(), torch.from_numpy(hs).bfloat16())


@pytest.mark.parametrize("g,bits", [(32, 8), (64, 4), (128, 8)])
def test_as_many_rows_as_a_plan_takes(wq, g, bits):
    R, Cin, Cout = 4194240, 128, 40
    print(g, bits, flush=True)
    rng = np.random.default_rng(g)
    plan, blob, ws, (wcodes, wscales), b = layer(wq, rng, R, Cin, Cout, g, bits)
    with pytest.raises(wq.WqError):
        wq.LinearPlan(R + 1, Cin, Cout, g)
    gen = torch.Generator(device="cuda").manual_seed(g)
    x = torch.randn((R, Cin), generator=gen, dtype=torch.bfloat16, device="cuda")
    y = torch.full((R, Cout), float("nan"), dtype=torch.bfloat16, device="cuda")
    plan.linear(x, blob, ws, y, activation="gelu")
    torch.cuda.synchronize()
    assert bool(y.isfinite().all())
    rows = sorted({0, 1, 127, 128, R // 2, R - 129, R - 128, R - 2, R - 1} | set(rng.integers(0, R, 40).tolist()))
    at = torch.tensor(rows, device="cuda")
    codes, scales = oracle.quantize_pixels(f32(x[at]), g)
    z, S = lb.product(codes, scales, wcodes, wscales, b, g)
    check_product(y[at], z, S, Cin // g, "gelu", False, None)

    def held():
        L = plan.layout
        xq = ws[L.ws_xq_off:L.ws_xq_off + R * Cin].view(torch.int8).view(Cin // L.kstep, 4, R, L.kstep // 4)[:, :, at]
        return xq.permute(2, 0, 1, 3).reshape(len(rows), Cin).cpu().numpy(), \
            ws[L.ws_sx_off:L.ws_sx_off + R * (Cin // g) * 4].view(torch.float32).view(Cin // g, R)[:, at].t().cpu().numpy()

    got = held()
    assert np.array_equal(got[0], codes) and np.array_equal(got[1], scales)
    plan.rms_norm_quantize(x, ws, eps=1e-5, out=x)
    torch.cuda.synchronize()
    _, codes, scales = lb.rms_norm_quantize(f32(x[at]), None, None, 1e-5, g)
    got = held()
    assert np.array_equal(got[0], codes) and np.array_equal(got[1], scales)

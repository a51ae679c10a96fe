"""Gradients in 16 bits are sums of codes that the matrix core forms directly: what it cuts off, to the last bit of the type.

Of each eight neighbours along the reduction the products are cut, towards zero, to multiples of 2^-13 of the largest one's power of two (that of its
two factors, each from 1 to 2 times a power of two).  The largest keeps all of its bits, so an eight loses less than 7 2^-13 of its largest."""
import pytest
import torch

from test_fp8_forms_gpu import U, quantized

pytestmark = pytest.mark.gpu


def cut_sum(A, B):
    """A [R][K] @ B [K][N] in 64 bits with the products of each eight of K cut as above."""
    out = torch.zeros((A.shape[0], B.shape[1]), dtype=torch.float64, device=A.device)
    power = lambda t: torch.where(t == 0, -1e4, torch.frexp(t)[1].double() - 1)   # noqa: E731
    for k in range(0, A.shape[1], 8):
        a, b = A[:, k:k + 8, None], B[None, k:k + 8, :]
        q = torch.exp2((power(a) + power(b)).amax(1, keepdim=True) - 13).clamp_min(1e-300)
        out += (torch.trunc(a * b / q) * q).sum(1)
    return out


def data(gen, kind, rows, C, O):
    """x [rows][C], dy [rows][O], w [O][C]"""
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")   # noqa: E731
    x, dy, w = r(rows, C), r(rows, O), r(O, C)
    if kind == "loud":      # one channel in fifty, and its weights, twenty times the others
        x[:, ::50] *= 20.0
        dy[:, ::50] *= 20.0
        w[::50] *= 20.0
    elif kind == "tokens":   # sizes from token to token as those of gradients
        x *= torch.exp(0.5 * r(rows, 1))
        dy *= torch.exp(1.5 * r(rows, 1))
        dy[31::32] = 0.0
    return x, dy, w


def check(got, A, B, K):
    want, S = cut_sum(A, B), A.abs() @ B.abs()
    half = torch.finfo(got.dtype).eps / 2
    e = (K + 16) * U * S
    bad = ~((got.double() - want).abs() <= e * 1.01 + half * (want.abs() + e) + torch.finfo(got.dtype).smallest_normal * half)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:5].tolist())
    full = A @ B
    assert bool(((want - full).abs() <= 7 * 2.0 ** -13 * S).all())
    return ((want - full).norm() / full.norm()).item()


# rows, Cin, Cout: a reduction of 1152 and one that ends inside an eight
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("kind", ["like", "loud", "tokens"])
def test_what_the_direct_sums_cut_off(wq, kind, dtype):
    gen = torch.Generator(device="cuda").manual_seed(21)
    for long in (1152, 1003):
        rows, C, O = 200, 136, long
        x, dy, w = data(gen, kind, rows, C, O)
        plan = wq.Fp8LinearPlan(rows, C, O, backward=True)
        blob, ws = plan.alloc_blob(), plan.alloc_workspace()
        plan.weight_prepare(w, None, blob)
        codes, s, _ = plan.blob_views(blob)
        W = codes.double() * s.double().repeat_interleave(128, 0)[:O].repeat_interleave(128, 1)[:, :C]
        dy = dy.to(dtype)
        dx = torch.empty((rows, C), dtype=dtype, device="cuda")
        plan.backward(None, dy, blob, ws, dx=dx)
        lost = [check(dx, quantized(dy.float(), 1), W, O)]
        x, dy, _ = data(gen, kind, long, C, 136)
        x, dy = x.to(dtype), dy.to(dtype)
        plan = wq.Fp8LinearPlan(long, C, 136, backward=True)
        dw = torch.empty((136, C), dtype=dtype, device="cuda")
        plan.backward(x, dy, None, plan.alloc_workspace(), dw=dw)
        lost.append(check(dw, quantized(dy.float(), 0).t().contiguous(), quantized(x.float(), 0), long))
        assert max(lost) <= (2e-5 if kind == "like" else 1.2e-4), lost

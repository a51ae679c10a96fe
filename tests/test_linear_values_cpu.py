"""Refusals of the linear layer's surroundings that a caller's memory manager can meet (no kernel is launched)."""
import pytest

from test_linear_block_cpu import INVALID, NOT_PREPARED, PTR, matmul_args, norm_args, quantize_args


@pytest.mark.parametrize("off", [1, 2, 4, 8])
def test_workspace_and_blob_are_aligned(wq, off):
    """Codes, scales and weights are moved in aligned pieces of 16 bytes."""
    plan, L = wq.LinearPlan(10, 128, 64, 32), wq.lib()
    assert L.wq_rms_norm_quantize(*norm_args(plan, ws=PTR + off)) == INVALID
    assert L.wq_linear_quantize(*quantize_args(plan, ws=PTR + off)) == INVALID
    assert L.wq_linear_matmul(*matmul_args(plan, ws=PTR + off)) == INVALID
    assert L.wq_linear_matmul(*matmul_args(plan, blob=PTR + off)) == INVALID
    assert L.wq_linear_matmul(*matmul_args(plan)) == NOT_PREPARED
    a = matmul_args(plan)
    for ws, blob, status in ((PTR + off, PTR, INVALID), (PTR, PTR + off, INVALID), (PTR, PTR, NOT_PREPARED)):
        assert L.wq_linear_forward(a[0], None, 10, 1, PTR, 128, blob, a[6], ws, a[4], 0, 0, None, 0, PTR, 64) == status

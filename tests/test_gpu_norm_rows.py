"""GPU parity of the layer norm where its backward has no rows, or more of them than blocks, in rows that a block does
not hold."""
import pytest
import torch

import paper_2606_07574_amd as b4
import tests._norm as reference
from tests.test_gpu_norm import EPS32, check, inputs

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("C", [524289, 1 << 20])
def test_no_rows(C, dtype):
    """Rows so wide that a share of them is one row: without rows the sums are zeros."""
    x, w = torch.empty(0, C, dtype=dtype, device="cuda"), torch.ones(C, dtype=dtype, device="cuda")
    y, mean, rstd = b4.norm_fwd(x, w, w)
    dx, dw, db = b4.norm_bwd(x, w, mean, rstd, x)
    torch.cuda.synchronize()
    assert y.shape == dx.shape == (0, C) and (dw == 0).all() and (db == 0).all()


def column_depth(B, C):
    """The sums over rows of more than 8192 values: a chain of a share's rows, then 16 parts of the shares, then these."""
    shares = max(1, min(2048 // ((C + 255) // 256), B))
    return -(-B // shares) + -(-shares // 16) + 16


@pytest.mark.parametrize("types", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)], ids=["f32", "mixed", "bf16", "f32bf16"])
@pytest.mark.parametrize("B,C", [(1100, 8200), (1100, 8201), (1100, 16392), (1100, 16385), (520, 65537)])
def test_long_rows(B, C, types, monkeypatch):
    """More rows than the blocks that take one each take at once."""
    monkeypatch.setattr(reference, "column_depth", column_depth)
    check(*inputs(B, C, *types, B + C), f"B={B} C={C} {types}")


def test_far_values():
    """What the header says of rows whose squares leave fp32's range: above it no spread is seen in front of them (rstd 0,
    y the bias, dx 0); with eps = 0 and deviations below it, NaN or infinities. The other rows do not change."""
    x, w, b, dy = inputs(6, 200, F32, F32, 3)
    plain = b4.norm_fwd(x, w, b, EPS32)
    far = x.clone()
    far[1] = x[1] * 1e20
    y, mean, rstd = b4.norm_fwd(far, w, b, EPS32)
    dx, dw, db = b4.norm_bwd(far, w, mean, rstd, dy)
    rest = [0, 2, 3, 4, 5]
    assert rstd[1] == 0 and torch.equal(y[1], b) and (dx[1] == 0).all()
    for got, want in zip((y, mean, rstd), plain):
        assert torch.equal(got[rest], want[rest])
    far[1] = x[1] * 1e-25
    y, mean, rstd = b4.norm_fwd(far, w, b, 0.0)
    assert not y[1].isfinite().any() and y[rest].isfinite().all()
    far[1] = x[1] * 1e15  # in range
    check(far, w, b, dy, "large but in range")

"""GPU parity of the layer norm where its backward has no rows, or more of them than blocks, in rows that a block does
not hold."""
import pytest
import torch

import paper_2606_07574_amd as b4

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

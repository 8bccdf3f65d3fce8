"""GPU parity of orth_step's direction for any momentum: G + momentum M with Nesterov's, M without, whatever the
momentum's sign."""
import pytest
import torch

import paper_2606_07574_amd as b4
from tests._orth import close
from tests.test_gpu_orth import matrices, step_ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("momentum", [-0.5, -1.0, -1.25, -0.0, 1.5])
@pytest.mark.parametrize("shape,w_dtype,g_dtype", [((24, 600), F32, F32), ((2, 600, 24), BF16, F32), ((150, 333), F32, BF16),
                                                   ((2, 200, 140), BF16, BF16)], ids=str)
def test_momentum_of_either_sign(shape, w_dtype, g_dtype, momentum, nesterov):
    W, G, M = matrices(shape, w_dtype, 1, "spread", 0.1), matrices(shape, g_dtype, 2, "spread"), matrices(shape, F32, 3, "spread")
    ref, M1, bound = step_ref(W, G, M, 0.5, momentum, nesterov, 0.1, 1.0, w_dtype == F32)
    b4.orth_step(W, G, M, 0.5, momentum, nesterov, 0.1, 1.0)
    close(W, ref.reshape(-1, *shape[-2:]), bound, f"{shape} {momentum} {nesterov}")
    assert ((M.double() - M1).abs() <= 2.0 ** -24 * M1.abs() + 1e-10).all()  # one fma of values below 0.1

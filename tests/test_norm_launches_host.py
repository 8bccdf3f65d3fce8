"""Which kernels the layer norm's backward launches, and on what, as the host decides it (no GPU needed)."""
import pytest

import paper_2606_07574_amd as b4
from tests._launches import launches

BWD = "pipippppppplllp"
MB = 1 << 28


@pytest.mark.parametrize("dtype", [b4.F32, b4.BF16], ids=["f32", "bf16"])
def test_no_rows_no_sums_read(dtype, tmp_path):
    """Without rows there is no workspace, and the sums are zeros that nothing is read for."""
    widths = (1, 16, 8192, 8193, 524288, 524289, 1 << 20)
    calls = [("birkhoff4_norm_bwd", BWD, [None, dtype, None, dtype, None, None, None, None, MB, 2 * MB, None, 0, 0, C, None])
             for C in widths]
    sizes = [("birkhoff4_norm_work", "lli", [0, C, dtype]) for C in widths]
    found = launches(calls + sizes, tmp_path)
    for C, (code, kernels) in zip(widths, found):
        assert code == 0 and [k[0] for k in kernels] == ["norm_join_kernel"], C
        assert kernels[0][2] == (2 * C + 63) // 64
        assert kernels[0][5:] == (0, 0), f"C={C}: reads {kernels[0][6]} rows of sums at {kernels[0][5]:#x}"
    assert all(size == 0 for size, _ in found[len(widths):])


def test_sums_that_are_there(tmp_path):
    """With rows, the join reads as many rows of sums as the workspace holds."""
    shapes = [(1, 1), (1, 1 << 20), (3, 524289), (5, 524288), (2, 8193), (700, 9000), (100000, 64), (300, 8192)]
    calls = []
    for B, C in shapes:
        calls.append(("birkhoff4_norm_work", "lli", [B, C, b4.BF16]))
        calls.append(("birkhoff4_norm_bwd", BWD, [MB << 10, b4.BF16, None, b4.F32, MB << 11, MB << 12, MB << 13, None, MB, 2 * MB, 3 * MB,
                                                  MB, B, C, None]))
    found = launches(calls, tmp_path)
    for (B, C), (size, _), (code, kernels) in zip(shapes, found[::2], found[1::2]):
        assert code == 0 and kernels[-1][0] == "norm_join_kernel"
        assert kernels[-1][5] == 3 * MB and kernels[-1][6] * 2 * C * 4 == size, (B, C)

"""Norm: 8-bit rows of values that pass fp32's range."""
import pytest
import torch

import paper_2512_22142_amd as cleave

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


@pytest.mark.parametrize("cols", [64, 100, 1000, 4096, 40000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_8_bit_rows_that_hold_an_infinity_are_nan(cols, dtype):
    """From finite x: an infinite weight, or a product with the weight beyond fp32."""
    x = torch.ones(3, cols, dtype=dtype, device="cuda")
    x[1, 5] = 0
    x[2] = 0                                            # 0 times infinity
    q, scales = torch.empty(x.shape, dtype=E4M3, device="cuda"), torch.empty(3, device="cuda")
    w = torch.ones(cols, device="cuda")
    w[cols // 2] = float("inf")
    cleave.rms_norm(x, w, q, scales=scales)
    assert torch.all(scales.isnan()) and torch.all(q.float().isnan())
    x[2], x[2, cols // 3] = 1, 8                        # 8 / rms is above 1.3
    w[cols // 2], w[cols // 3] = 1, 3e38
    cleave.rms_norm(x, w, q, scales=scales)
    assert scales[2].isnan() and torch.all(q[2].float().isnan())
    for row in (0, 1):                                  # 3e38 itself is finite
        assert scales[row].isfinite() and q[row, cols // 3].float() == 448

"""Rows of as many values as the quantisation takes (2^30: 4 GB of fp32): positions whose byte offsets pass 31 and 32 bits."""
import numpy as np
import pytest
import torch

from oracle import operators as O
from tests.test_gpu_quantized import DTYPES, b  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [2 ** 29 + 40, 2 ** 30 - 3, 2 ** 30])
def test_one_row(b, dtype, cols):  # noqa: F811
    at = np.unique([0, 9, 2 ** 29 - 9, 2 ** 29 - 1, 2 ** 29, 2 ** 29 + 13, cols // 2 + 5, cols - 9, cols - 8, cols - 1])
    values = np.linspace(-1.75, 2.0, at.size).astype(np.float32)
    ld = (cols + 15) // 16 * 16
    x, q = torch.zeros(1, ld, dtype=dtype, device="cuda")[:, :cols], torch.full((1, ld), 55, dtype=torch.int8, device="cuda")
    scale, where = torch.full((1,), -1.0, device="cuda"), torch.from_numpy(at).cuda()
    x[0, where] = torch.from_numpy(values).cuda().to(dtype)
    b.quantize_rows(x, q[:, :cols], scale)
    want, ws = O.quantize_rows(x[0, where].float().cpu().numpy()[None])          # the other values are 0
    assert np.array_equal(q[0, where].cpu().numpy(), want[0]) and scale.item() == ws[0]
    assert torch.count_nonzero(q[:, :cols]).item() == np.count_nonzero(want) and torch.all(q[:, cols:] == 55)

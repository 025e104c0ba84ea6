"""Rows of 8-bit whole numbers at the widest that heta_linear_rows_i8 takes: a step behind the last columns is past 2^31."""
import pytest
import torch

import paper_2408_09697_amd as heta
from tests.test_gpu_i8 import BF16, I8, U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [2 ** 31 - 1024, 2 ** 31 - 2048 + 5])
def test_widest_row(d):
    """Columns around each power of two and at the end differ; what lies behind the row stays."""
    x, q = torch.full((1, d + 64), 1.0, dtype=BF16, device="cuda"), torch.full((1, d + 64), 99, dtype=I8, device="cuda")
    x[0, 0], x[0, d - 1], x[0, d:] = -127.0, 3.0, float("nan")
    for at in (2 ** 30, 2 ** 31 - 4096, d - 2048, d - 9, d - 8):
        x[0, at] = 50.0
    scale = torch.empty(1, device="cuda")
    heta.heta_linear_rows_i8(x[:, :d], q[:, :d], scale)
    assert abs(float(scale[0]) - 1) <= 2 * U
    assert (q[0, d:] == 99).all()
    for i in range(0, d, 1 << 28):  # values are whole already: 127 / 127 of each
        assert torch.equal(q[0, i:min(d, i + (1 << 28))], x[0, i:min(d, i + (1 << 28))].to(I8))
    del x, q
    torch.cuda.empty_cache()

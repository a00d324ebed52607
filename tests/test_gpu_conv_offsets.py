"""Offsets and sizes of the convolution layers whose sums or products would not fit 64 bits are refused."""
import pytest
import torch

from paper_1705_09056_b200 import binding, workloads as wl
from tests.gpu_util import GpuRun

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w_off,b_off", [(2 ** 63 - 1, 0), (0, 2 ** 63 - 1), (2 ** 63 - 432, 0), (0, 2 ** 63 - 16), (-1, 0), (0, -1)])
def test_blocks_far_outside_the_parameter_row(w_off, b_off):
    g = GpuRun(2, 16 * 3 * 9 + 16, wl.topology("ring", 2), 0.1)
    x, y = torch.zeros(2 * 8 * 3 * 64, device="cuda"), torch.zeros(2 * 8 * 16 * 64, device="cuda")
    lib, h = g.ctx._lib, g.ctx._h
    p = lambda t: t.data_ptr()                                                   # noqa: E731
    assert lib.dpsgd_conv3x3_forward(h, p(x), 8, 3, 8, 8, 16, 1, w_off, b_off, 1, p(y)) == binding.ERR_ARG
    assert lib.dpsgd_conv3x3_backward(h, p(x), p(y), p(y), 8, 3, 8, 8, 16, 1, w_off, b_off, 1, 0) == binding.ERR_ARG
    g.close()


def test_filter_counts_whose_product_does_not_fit():
    g = GpuRun(1, 64, wl.topology("ring", 1), 0.1)
    x = torch.zeros(1024, device="cuda")
    lib, h, big = g.ctx._lib, g.ctx._h, 2 ** 31 - 16
    assert lib.dpsgd_conv3x3_backward(h, x.data_ptr(), x.data_ptr(), x.data_ptr(), 1, big, 8, 8, big, 1, 0, 0, 1, 0) == binding.ERR_ARG
    g.close()

"""8-bit layers at the edges of what they accept: padding, special values, buffers' surroundings, sizes, workspaces."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as fo
from paper_1705_09056_b200 import binding, workloads as wl
from tests.gpu_util import GpuRun
from tests.test_gpu_fp8_layers import Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,B,K,O", [(1, 40, 256, 130), (2, 3, 300, 1001), (12, 300, 700, 700)])
def test_checkpoint_padding_of_rows_with_nan(n, B, K, O):
    """The checkpoint of the forward product is that of its fp32 result byte for byte, padding included, in rows whose
    input holds a NaN too (tiles of one CTA and of pairs)."""
    l = Layer(n, B, K, O)
    q = l.x8.q.clone()
    q[0, 1, 3] = q[-1, B - 1, K - 1] = 0x7F
    x8 = binding.Ckpt8(q, l.x8.e, K)
    y, c = torch.empty((n, B, O), device="cuda"), l.ctx.ckpt8_empty((n, B, O))
    c.q.fill_(0x55), c.e.fill_(0x55)
    l.ctx.fp8_linear_forward(x8, l.w8, b_off=l.b_off, out=y, ckpt=c)
    assert bool(torch.isnan(y[0, 1]).all()) and bool(torch.isnan(y[-1, B - 1]).all()) and int(torch.isnan(y).sum()) == 2 * O
    ref = l.ctx.ckpt8_save(y)
    assert torch.equal(c.q, ref.q) and torch.equal(c.e, ref.e)
    assert not c.q[..., O:].any()
    l.close()


@pytest.mark.parametrize("off", [2 ** 63 - 1, 2 ** 63 - 16, 2 ** 62, -2, -2 ** 63])
def test_offsets_near_the_ends_of_64_bits_are_refused(off):
    """offset + size must not wrap round on its way to the comparison with N."""
    l = Layer(2, 4, 32, 16)
    y, dy = torch.zeros(2, 4, 16, device="cuda"), torch.zeros(2, 4, 16, device="cuda")
    for call in (lambda: l.ctx.fp8_linear_forward(l.x8, l.w8, b_off=off, out=y),
                 lambda: l.ctx.fp8_linear_backward(l.x8, l.w8, dy, w_off=0, b_off=off),
                 lambda: l.ctx.fp8_linear_backward(l.x8, l.w8, dy, w_off=off),
                 lambda: l.ctx.fp8_weights(off, 16, 32)):
        with pytest.raises(binding.DpsgdError):
            call()
    l.close()

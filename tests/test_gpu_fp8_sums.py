"""How the 8-bit products add, seen on sums of terms of one sign.

An MMA that adds to an accumulator truncates it, so m MMAs before it is handed over lose in proportion to the accumulator
each of them finds: (1 + ... + m) / m = (m + 1) / 2 units on an even growth, whatever the unit is.  What follows in fp32
registers rounds to nearest, either way, and loses nothing on average.
"""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as fo
from paper_1705_09056_b200 import workloads as wl
from tests.gpu_util import GpuRun

pytestmark = pytest.mark.gpu


class Net:
    """One layer without bias, weights and input as values that 8 bits hold."""

    def __init__(self, x, w):
        (self.B, self.K), self.O = x.shape, w.shape[0]
        self.g = GpuRun(1, w.size, wl.topology("ring", 1), 0.1, X=w.reshape(1, -1))
        self.ctx = self.g.ctx
        self.x8 = self.ctx.ckpt8_save(torch.from_numpy(x[None]).cuda())
        self.w8 = self.ctx.fp8_weights(0, self.O, self.K)
        self.xv = fo.load(*fo.save(x), self.K)
        self.wv = fo.weight_values(*fo.weights(w), self.K)
        self.ref = self.xv @ self.wv.T

    def close(self):
        self.ctx.sync()
        self.g.close()


@pytest.mark.parametrize("B,K,O", [(64, 2048, 256), (32, 784, 1024), (100, 4097, 130)])
def test_sums_behind_a_checkpoint_are_handed_over_every_eight_mmas(B, K, O):
    """Up to 128 rows.  An fp32 result alone is handed over every 16: 17 / 2 units against 9 / 2, a ratio of 0.53."""
    rng = np.random.default_rng(B + K)
    n = Net(np.abs(rng.standard_normal((B, K))).astype(np.float32), np.abs(rng.standard_normal((O, K))).astype(np.float32))
    lost = []
    for ckpt in (None, n.ctx.ckpt8_empty((1, B, O))):
        y = torch.empty((1, B, O), device="cuda")
        n.ctx.fp8_linear_forward(n.x8, n.w8, out=y, ckpt=ckpt)
        lost.append(float(((n.ref - y[0].cpu().numpy().astype(np.float64)) / n.ref).mean()))
    assert 0.0 < lost[0] < 2.0 ** -20 and lost[1] <= 0.75 * lost[0], lost
    n.close()

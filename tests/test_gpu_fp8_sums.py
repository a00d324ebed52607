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


# 128 MMAs lose at most a unit each of the accumulator they find: (1 + ... + 128) / 128 * 2^-23 of the sum of magnitudes
COARSE = 64.5 * 2.0 ** -23


def long_rows(rows, K, cancel, seed):
    """Positive rows; with `cancel` the second half repeats the first (the other factor there has the opposite sign)."""
    v = np.abs(np.random.default_rng(seed).standard_normal((rows, K))).astype(np.float32)
    if cancel:
        v[:, K // 2:] = v[:, :K // 2]
    return v


@pytest.mark.parametrize("K", [16384, 65536])
@pytest.mark.parametrize("cancel", [False, True])
def test_bf16_results_of_long_contractions(K, cancel):
    """bf16 rounds to nearest: half a step, 2^-9 of a value, and on average over R values 2^-8 / sqrt(12 R) either way."""
    B, O = 64, 512
    x, w = long_rows(B, K, cancel, K), long_rows(O, K, cancel, K + 1)
    if cancel:
        w[:, K // 2:] *= -1.0
    n = Net(x, w)
    y = n.ctx.fp8_linear_forward(n.x8, n.w8, dtype=torch.bfloat16)[0].float().cpu().numpy().astype(np.float64)
    S = np.abs(n.xv) @ np.abs(n.wv).T
    if cancel:
        assert not n.ref.any() and (np.abs(y) <= COARSE * S * (1 + 2.0 ** -8)).all(), np.abs(y / S).max()
    else:
        assert (np.abs(y - n.ref) <= COARSE * S + 2.0 ** -8 * n.ref).all()
        assert abs(((n.ref - y) / n.ref).mean()) <= COARSE + 4 * 2.0 ** -8 / (12 * B * O) ** 0.5
    n.close()


def test_bf16_input_gradients_of_many_outputs():
    """dx adds over the outputs of the layer."""
    B, K, O = 64, 128, 65536
    w, dy = long_rows(O, K, False, 1), long_rows(B, O, False, 2)
    n = Net(long_rows(B, K, False, 3), w)
    dx = torch.empty((1, B, K), dtype=torch.bfloat16, device="cuda")
    n.ctx.fp8_linear_backward(n.x8, n.w8, torch.from_numpy(dy[None]).cuda(), w_off=0, dx=dx)
    ref = fo.load(*fo.save(dy), O) @ n.wv
    got = dx[0].float().cpu().numpy().astype(np.float64)
    assert (np.abs(got - ref) <= COARSE * ref + 2.0 ** -8 * ref).all()
    assert abs(((ref - got) / ref).mean()) <= COARSE + 4 * 2.0 ** -8 / (12 * B * K) ** 0.5
    n.close()

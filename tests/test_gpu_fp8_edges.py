"""8-bit layers at the edges of what they accept: padding, special values, buffers' surroundings, sizes, workspaces."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as fo
from paper_1705_09056_b200 import binding, workloads as wl
from tests.gpu_util import GpuRun
from tests.test_gpu_fp8_layers import PAIRS, SHAPES, TOL_BF16, TOL_SUM, Layer

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


def free_bytes():
    torch.cuda.synchronize()
    return torch.cuda.mem_get_info()[0]


def test_set_model_allocates_all_that_a_gradient_needs():
    """A hidden layer wider than the later ones: no allocation, hence no device synchronisation, inside the gradient."""
    w = wl.mlp_workload(n=4, dims=(64, 1024, 2048, 10), m=64, batch=512, gamma=0.05, seed=1)
    A, y = w.A.cuda(), w.y.cuda()
    for again in (False, True):                      # the first context also loads the kernels
        run = GpuRun(4, w.N, w.csr(), w.gamma, seed=1, X=np.tile(w.x0.numpy(), (4, 1)))
        run.ctx.set_model(w.model, w.dims, 0.0, 512, 3)
        run.ctx.set_data(A, y)
        before = free_bytes()
        run.ctx.grad(0)
        assert not again or free_bytes() == before
        run.ctx.sync()
        run.close()


def test_reserve_allocates_what_a_backward_needs():
    for again in (False, True):
        l = Layer(3, 300, 1000, 1004)
        dy, dx = torch.randn(3, 300, 1004, device="cuda"), torch.empty(3, 300, 1000, device="cuda")
        l.ctx.fp8_reserve(301, 1000, 1010)           # layers of up to this size
        before = free_bytes()
        l.ctx.fp8_linear_backward(l.x8, l.w8, dy, w_off=0, b_off=l.b_off, dx=dx)
        assert not again or free_bytes() == before
        l.close()


def test_reserve_refusals():
    l = Layer(1, 2, 32, 16)
    r, h = l.ctx._lib.dpsgd_fp8_reserve, l.ctx._h
    assert r(None, 1, 1, 1) == r(h, 0, 1, 1) == r(h, 1, -1, 1) == r(h, 1, 1, 0) == binding.ERR_ARG
    assert r(h, 1, 65537, 1) == r(h, (1 << 20) + 1, 1, 1) == binding.ERR_UNSUPPORTED
    assert r(h, 1, 1, 1) == binding.OK
    l.close()


def test_captured_backward_keeps_its_workspace():
    """Without a reserved workspace a capture is refused before it records anything; a graph that was captured computes
    the same after a larger layer has made the workspace grow and others have taken the memory that is free."""
    n, B, K, O = 2, 150, 520, 600
    l = Layer(n, B, K, O)
    s = torch.cuda.Stream()
    l.ctx.bind(l.g.X0, l.g.X1, l.g.G, stream=s)
    dy, dx = torch.randn(n, B, O, device="cuda"), torch.empty(n, B, K, device="cuda")
    call = lambda: l.ctx.fp8_linear_backward(l.x8, l.w8, dy, w_off=0, b_off=l.b_off, dx=dx)   # noqa: E731
    torch.cuda.synchronize()
    empty = torch.cuda.CUDAGraph()
    with torch.cuda.graph(empty, stream=s):
        with pytest.raises(binding.DpsgdError) as e:
            call()
        dy.add_(0.0)                                 # the capture is still intact
    assert "reserve" in str(e.value)
    l.ctx.fp8_reserve(B, K, O)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
    graph.replay()
    torch.cuda.synchronize()
    G, D = l.g.G.clone(), dx.clone()
    for i in range(n):
        ref, _ = fo.backward(l.xv[i], l.wv[i], dy[i].cpu().numpy(), None)
        assert np.abs(D[i].cpu().numpy() - ref[2]).max() <= 1e-4 * np.abs(ref[2]).max()
    l.ctx.fp8_reserve(16 * B, K, O)                  # grows
    junk = torch.full((256 << 20,), 0x7F, dtype=torch.uint8, device="cuda")
    l.g.G.fill_(3.0), dx.fill_(3.0)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(l.g.G[:, :l.N], G[:, :l.N]) and torch.equal(dx, D)
    assert bool((junk == 0x7F).all())
    del graph, empty
    l.close()


@pytest.mark.parametrize("precision", [-1, 4, 8, 2 ** 31 - 1])
def test_precisions_that_do_not_exist_are_refused(precision):
    """3 stands for 8-bit layers; a number beside the four must not run as some other precision.  Linear models have none."""
    w = wl.mlp_workload(n=2, dims=(16, 20, 4), m=16, batch=4, gamma=0.05, seed=1)
    run = GpuRun(2, w.N, w.csr(), w.gamma)
    with pytest.raises(binding.DpsgdError) as e:
        run.ctx.set_model(w.model, w.dims, 0.0, 4, precision)
    assert e.value.status == binding.ERR_ARG
    for ok in (0, 1, 2, 3):
        run.ctx.set_model(w.model, w.dims, 0.0, 4, ok)
    run.close()
    lin = GpuRun(2, 16, wl.topology("ring", 2), 0.1)
    lin.ctx.set_model(binding.MODEL_LSQ, [16], 0.0, 4, precision)
    lin.close()


@pytest.mark.parametrize("B", [65, 128, 129])
def test_weight_gradient_beyond_l2_on_both_sides_of_the_sample_limit(B):
    """546 MB of gradient, two k-blocks of samples on pairs of CTAs and three on single ones; first and last node."""
    n, K, O = 70, 1500, 1300
    N = O * K
    ld = wl.padded_ld(N)
    X = torch.zeros(n, ld, device="cuda")
    X[:, :N].normal_()
    G = torch.full_like(X, 3.0)
    ctx = binding.Dpsgd(n, N, *wl.ring(n), gamma=0.1)
    ctx.bind(X, torch.zeros_like(X), G)
    x, dy = torch.randn(n, B, K, device="cuda"), torch.randn(n, B, O, device="cuda")
    ctx.fp8_linear_backward(ctx.ckpt8_save(x), ctx.fp8_weights(0, O, K), dy, w_off=0)
    ctx.sync()
    assert bool((G[:, N:] == 3.0).all())
    for i in (0, n - 1):
        xv, d8 = fo.load(*fo.save(x[i].cpu().numpy()), K), fo.load(*fo.save(dy[i].cpu().numpy()), O)
        got = G[i, :N].view(O, K).cpu().numpy().astype(np.float64)
        assert (np.abs(got - d8.T @ xv) <= TOL_SUM * (np.abs(d8).T @ np.abs(xv))).all()
    ctx.close()


# bf16 results alone choose among four tiles; the last three are shared by pairs of CTAs, ragged in every direction and with
# two tiles per pair
@pytest.mark.parametrize("n,B,K,O", SHAPES + PAIRS + [(24, 256, 2100, 768), (18, 1000, 1100, 500), (9, 257, 4097, 1025)])
def test_forward_with_a_bf16_result_alone(n, B, K, O):
    l = Layer(n, B, K, O, off=3)
    y = l.ctx.fp8_linear_forward(l.x8, l.w8, b_off=l.b_off, relu=True, dtype=torch.bfloat16).float().cpu().numpy().astype(np.float64)
    ref, scale = l.forward(True)
    assert (np.abs(y - ref) <= TOL_SUM * scale + TOL_BF16 * np.abs(ref)).all()
    y2 = torch.full((n, B, O), 7.0, dtype=torch.bfloat16, device="cuda")
    l.ctx.fp8_linear_forward(l.x8, l.w8, b_off=l.b_off, relu=True, out=y2)
    assert np.array_equal(y2.float().cpu().numpy().astype(np.float64), y)                # reproducible
    l.close()

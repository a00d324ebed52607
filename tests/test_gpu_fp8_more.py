"""8-bit layers: derivatives against differences with bounds far below them, surroundings of every buffer, special values,
checkpoints byte for byte, and the largest sizes."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as fo
from paper_1705_09056_b200 import binding, workloads as wl
from tests.gpu_util import GpuRun
from tests.test_gpu_fp8_layers import PAIRS, SHAPES, TOL_BF16, TOL_SUM, Layer

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- differences

def test_gradients_agree_with_differences_of_the_forward():
    """The layer without ReLU is linear in each byte of x, each byte of W and each bias.  A byte goes from 448 to -448, so
    that the change is not small beside the other terms; y is subtracted element by element in 64 bits.  Each of two
    sums is off by TOL_SUM / 2 of its terms at most, hence a difference quotient by TOL_SUM * sum |terms| / change."""
    n, B, K, O = 1, 9, 160, 96
    l = Layer(n, B, K, O)
    dyv = fo.load(*fo.save(l.rng.standard_normal((B, O)).astype(np.float32)), O)
    dy = torch.from_numpy(dyv.astype(np.float32).reshape(n, B, O)).cuda()
    dx = torch.empty((n, B, K), device="cuda")
    l.ctx.fp8_linear_backward(l.x8, l.w8, dy, w_off=0, b_off=l.b_off, dx=dx)
    dx = dx[0].cpu().numpy().astype(np.float64)
    gw = l.g.G[0, :O * K].view(O, K).cpu().numpy().astype(np.float64)
    gb = l.g.G[0, l.b_off:l.b_off + O].cpu().numpy().astype(np.float64)
    y = lambda x8, w8: l.ctx.fp8_linear_forward(x8, w8, b_off=l.b_off)[0].cpu().numpy().astype(np.float64)   # noqa: E731
    xe, we = l.x8.e.cpu().numpy().astype(np.float64), l.w8.e.cpu().numpy().astype(np.float64)

    def bytes_of(q, at):
        out = []
        for b in (0x7E, 0xFE):
            c = q.clone()
            c[at] = b
            out.append(c)
        return out

    for b, k in ((0, 0), (3, 131), (8, 159)):
        k = int(np.abs(dx[b, k // 128 * 128:k // 128 * 128 + 32]).argmax()) + k // 128 * 128     # a clear derivative nearby
        step = 2 * 448 * 2.0 ** (xe[0, b, k // 128] - 127)
        up, dn = (y(binding.Ckpt8(q, l.x8.e, K), l.w8) for q in bytes_of(l.x8.q, (0, b, k)))
        num = ((up - dn) * dyv).sum() / step
        terms = np.abs(l.xv[0, b]) @ np.abs(l.wv[0]).T + step * np.abs(l.wv[0, :, k]) + np.abs(l.bias[0])
        bound = TOL_SUM * (np.abs(dyv[b]) @ terms / step + np.abs(dyv[b]) @ np.abs(l.wv[0, :, k]))
        assert bound <= 0.02 * abs(dx[b, k]) and abs(num - dx[b, k]) <= bound, (num, dx[b, k], bound)
    for o, k in ((0, 0), (50, 140), (95, 159)):
        k = int(np.abs(gw[o, k // 128 * 128:k // 128 * 128 + 32]).argmax()) + k // 128 * 128
        step = 2 * 448 * 2.0 ** (we[0, o // 128, k // 128] - 127)
        up, dn = (y(l.x8, binding.Fp8Weights(q, l.w8.e, K)) for q in bytes_of(l.w8.q, (0, o, k)))
        num = ((up - dn) * dyv).sum() / step
        terms = np.abs(l.xv[0]) @ np.abs(l.wv[0, o]) + step * np.abs(l.xv[0, :, k]) + np.abs(l.bias[0, o])
        bound = TOL_SUM * (np.abs(dyv[:, o]) @ terms / step + np.abs(dyv[:, o]) @ np.abs(l.xv[0, :, k]))
        assert bound <= 0.02 * abs(gw[o, k]) and abs(num - gw[o, k]) <= bound, (num, gw[o, k], bound)
    X = l.ctx.current()
    for o in (0, 50, 95):
        keep = float(X[0, l.b_off + o])
        X[0, l.b_off + o] = keep + 1.0
        up = y(l.x8, l.w8)
        X[0, l.b_off + o] = keep - 1.0
        dn = y(l.x8, l.w8)
        X[0, l.b_off + o] = keep
        # the same sums, so that only the last additions round: half a unit of y, of the shifted bias and of the sum each
        bound = 4 * 2.0 ** -24 * np.abs(dyv[:, o]) @ (np.abs(up[:, o]) + np.abs(dn[:, o]) + abs(keep) + 1.0)
        num = ((up - dn) * dyv).sum() / 2
        assert bound <= 0.02 * abs(gb[o]) and abs(num - gb[o]) <= bound, (num, gb[o], bound)
    l.close()


# ---------------------------------------------------------------- surroundings

class Guards:
    """Tensors cut out of larger buffers of marker bytes, which check() expects unharmed."""

    def __init__(self):
        self.kept = []

    def empty(self, shape, dtype=torch.uint8, shift=0):
        size = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        at = 512 + shift
        flat = torch.full((at + size + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        self.kept.append((flat, at, size))
        return flat[at:at + size].view(dtype).view(shape)

    def ckpt(self, n, B, d):
        return binding.Ckpt8(self.empty((n, B, -(-d // 16) * 16)), self.empty((n, B, -(-d // 512) * 4), shift=4), d)

    def check(self):
        torch.cuda.synchronize()
        for flat, at, size in self.kept:
            assert bool((flat[:at] == 0xA5).all()) and bool((flat[at + size:] == 0xA5).all())


@pytest.mark.parametrize("n,B,K,O", SHAPES + PAIRS)
@pytest.mark.parametrize("dtype,shift", [(torch.float32, 4), (torch.bfloat16, 2), (torch.bfloat16, 16)])
def test_nothing_is_written_beside_the_results(n, B, K, O, dtype, shift):
    """Every buffer at an odd place between marker bytes; parameter and gradient blocks between other columns."""
    off = 5
    l = Layer(n, B, K, O, off=off)
    gd = Guards()
    x = torch.randn(n, B, K, device="cuda").to(dtype)
    x8 = l.ctx.ckpt8_save(x, out=gd.ckpt(n, B, K))
    l.ctx.ckpt8_load(x8, out=gd.empty((n, B, K), dtype, shift))
    w8 = l.ctx.fp8_weights(off, O, K, out=binding.Fp8Weights(gd.empty((n, O, -(-K // 16) * 16)),
                                                              gd.empty((n, -(-O // 128), -(-K // 512) * 4), shift=4), K))
    y8 = gd.ckpt(n, B, O)
    l.ctx.fp8_linear_forward(x8, w8, b_off=l.b_off, relu=True, out=gd.empty((n, B, O), dtype, shift), ckpt=y8)
    l.ctx.fp8_linear_forward(x8, w8, b_off=l.b_off, out=gd.empty((n, B, O), dtype, shift))
    dy = torch.randn(n, B, O, device="cuda").to(dtype)
    l.g.G.fill_(3.0)
    l.ctx.fp8_linear_backward(x8, w8, dy, w_off=off, b_off=l.b_off, gate=y8.q, dx=gd.empty((n, B, K), dtype, shift))
    gd.check()
    l.g.check_pads()
    assert bool((l.g.G[:, :off] == 3.0).all()) and bool((l.g.G[:, l.N:] == 3.0).all())
    assert bool((x8.q[..., K:] == 0).all()) and bool((w8.q[..., K:] == 0).all()) and bool((y8.q[..., O:] == 0).all())
    l.close()


@pytest.mark.parametrize("n,B,K,O", SHAPES + PAIRS)
@pytest.mark.parametrize("relu", [False, True])
def test_checkpoint_of_the_forward_is_that_of_its_result(n, B, K, O, relu):
    """q and e, padding included, byte for byte: the fp32 result of the same call is rounded once, by the definition."""
    l = Layer(n, B, K, O)
    y, c = torch.empty((n, B, O), device="cuda"), l.ctx.ckpt8_empty((n, B, O))
    l.ctx.fp8_linear_forward(l.x8, l.w8, b_off=l.b_off, relu=relu, out=y, ckpt=c)
    ref = l.ctx.ckpt8_save(y)
    assert torch.equal(c.q, ref.q) and torch.equal(c.e, ref.e)
    l.close()


# ---------------------------------------------------------------- special values

LOWEST = float(np.finfo(np.float32).min)


def agree(got, ref, scale, rel=0.0):
    """Equal NaN and infinities, the rest within the bound of a sum.  Where the sum of magnitudes is beyond fp32, sums in
    fp32 may overflow on their way whatever their order: an element is within its bound there, or not finite."""
    got = got.astype(np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        ref32 = ref.astype(np.float32).astype(np.float64)
        near = np.abs(got - ref) <= TOL_SUM * scale + rel * np.abs(ref) + 2.0 ** -140
    beyond = np.isfinite(scale) & (scale >= np.finfo(np.float32).max)
    assert (near | ~np.isfinite(got))[beyond].all()
    same = np.where(np.isnan(ref32), np.isnan(got), np.where(np.isinf(ref32), got == ref32, near))
    assert same[~beyond].all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gated", [False, True])
def test_backward_of_special_output_gradients(dtype, gated):
    """NaN and infinities reach the row of dx and the row of gW that they belong to, and only those; the type's lowest value
    stays finite; behind a closed gate (zero, negative zero, NaN) all of them count as zero."""
    n, B, K, O = 2, 70, 200, 300
    l = Layer(n, B, K, O)
    l.x8 = l.ctx.ckpt8_save(torch.from_numpy((l.xv * 2.0 ** -12).astype(np.float32)).cuda())     # the lowest times x is finite
    xv = fo.load(*fo.save((l.xv * 2.0 ** -12).astype(np.float32).reshape(n * B, K)), K).reshape(n, B, K)
    dy = l.rng.standard_normal((n, B, O)).astype(np.float32)
    lowest = LOWEST if dtype == torch.float32 else float(torch.finfo(torch.bfloat16).min)
    for i, b, o, v in ((0, 3, 5, np.nan), (0, 40, 250, np.inf), (0, 41, 299, -np.inf), (1, 0, 0, lowest), (1, 69, 200, -lowest)):
        dy[i, b, o] = v
    t = torch.from_numpy(dy).to(dtype).cuda()
    d = t.float().cpu().numpy()
    gate = None
    if gated:
        gate = torch.full((n, B, -(-O // 16) * 16), 0x38, dtype=torch.uint8, device="cuda")
        for (i, b, o), byte in {(0, 3, 5): 0x00, (0, 40, 250): 0x80, (1, 0, 0): 0x7F, (0, 9, 9): 0xFF, (0, 8, 8): 0xB8}.items():
            gate[i, b, o] = byte
            d[i, b, o] = 0.0                         # 0xB8 is -1: a ReLU output never is, but it is not above zero
    dx = torch.empty((n, B, K), dtype=dtype, device="cuda")
    l.ctx.fp8_linear_backward(l.x8, l.w8, t, w_off=0, b_off=l.b_off, gate=gate, dx=dx)
    for i in range(n):
        d8 = fo.load(*fo.save(d[i]), O)
        with np.errstate(invalid="ignore", over="ignore"):
            ref = (d8.T @ xv[i], d[i].astype(np.float64).sum(0), d8 @ l.wv[i])
            # a row that holds the lowest value loses its small terms against it: scale = sum of magnitudes
            scale = (np.abs(d8).T @ np.abs(xv[i]), np.abs(d[i].astype(np.float64)).sum(0), np.abs(d8) @ np.abs(l.wv[i]))
        agree(l.g.G[i, :O * K].view(O, K).cpu().numpy(), ref[0], scale[0])
        agree(l.g.G[i, l.b_off:l.b_off + O].cpu().numpy(), ref[1], scale[1])
        agree(dx[i].float().cpu().numpy(), ref[2], scale[2], rel=0.0 if dtype == torch.float32 else TOL_BF16)
    assert int(torch.isnan(l.g.G).any(1).sum()) == 1
    l.close()


@pytest.mark.parametrize("B", [40, 300])
def test_forward_of_special_values(B):
    """Rows whose mask left the lowest value, infinite biases, a weight block whose scale is the largest."""
    n, K, O = 12, 256, 520
    l = Layer(n, B, K, O)
    x = l.rng.standard_normal((n, B, K)).astype(np.float32)
    x[0, 3, :] = LOWEST * np.float32(2.0 ** -4)
    x[0, 5, 130:] = LOWEST
    x[1, 7, :] = 0.0
    x8 = l.ctx.ckpt8_save(torch.from_numpy(x).cuda())
    xv = fo.load(*fo.save(x.reshape(n * B, K)), K).reshape(n, B, K)
    X = l.ctx.current()
    X[2, 128 * K:256 * K] *= 2.0 ** 100
    X[:, l.b_off + 1], X[:, l.b_off + 500] = float("inf"), -float("inf")
    Xh = X.cpu().numpy()
    w8 = l.ctx.fp8_weights(0, O, K)
    y, c = torch.empty((n, B, O), device="cuda"), l.ctx.ckpt8_empty((n, B, O))
    l.ctx.fp8_linear_forward(x8, w8, b_off=l.b_off, out=y, ckpt=c)
    for i in (0, 1, 2, n - 1):
        wv = fo.weight_values(*fo.weights(Xh[i, :O * K].reshape(O, K)), K)
        bias = Xh[i, l.b_off:l.b_off + O].astype(np.float64)
        ref, scale = fo.forward(xv[i], wv, bias, False)
        agree(y[i].cpu().numpy(), ref, scale)
    ref = l.ctx.ckpt8_save(y)
    assert torch.equal(c.q, ref.q) and torch.equal(c.e, ref.e)
    want = torch.where(y < 0, torch.zeros_like(y), y)                            # the same sums through ReLU; NaN stays
    l.ctx.fp8_linear_forward(x8, w8, b_off=l.b_off, relu=True, out=y, ckpt=c)
    assert bool(((y == want) | (y.isnan() & want.isnan())).all())
    ref = l.ctx.ckpt8_save(y)
    assert torch.equal(c.q, ref.q) and torch.equal(c.e, ref.e)
    assert bool((c.q[:, :, 1] == 0x7F).all()) and bool((c.q[:, :, 500] == 0).all())
    l.close()


# ---------------------------------------------------------------- a whole network whose sums meet no tie

@pytest.mark.parametrize("n,dims,m,B", [(3, (20, 33, 7), 40, 5), (5, (16, 10), 30, 8), (2, (130, 70, 3), 33, 1), (2, (64, 96, 80, 10), 50, 16)])
def test_small_networks_match_the_oracle_to_the_last_sums(n, dims, m, B):
    """About 2^-20 of the values that are rounded to 8 bits lie within a rounding of a tie, and 2^-12 of those that are
    rounded to bf16: none of the few hundred to thousand here is expected to, one of the latter may (2^-8 of one error)."""
    w = wl.mlp_workload(n=n, dims=dims, m=m, batch=B, gamma=0.05, seed=11)
    run = GpuRun(n, w.N, w.csr(), w.gamma, seed=3, X=np.tile(w.x0.numpy(), (n, 1)))
    run.ctx.set_model(w.model, w.dims, 0.0, B, 3)
    A, y = w.A.cuda(), w.y.cuda()
    run.ctx.set_data(A, y)
    idx = run.ctx.sample(4).cpu().numpy()
    run.ctx.grad(4)
    G = run.g()
    for i in range(n):
        ref = fo.grad_mlp8(w.x0.numpy(), dims, w.A[i].numpy(), w.y[i].numpy(), idx[i])
        assert np.linalg.norm(G[i] - ref) <= 2.0 ** -13 * np.linalg.norm(ref)
    run.close()


# ---------------------------------------------------------------- the largest sizes

def test_widest_rows():
    rng = np.random.default_rng(0)
    g = GpuRun(1, 32, wl.topology("ring", 1), 0.1)
    x = (rng.standard_normal((3, 65536)) * np.exp(rng.standard_normal(65536))).astype(np.float32)
    c = g.ctx.ckpt8_save(torch.from_numpy(x).cuda())
    q, e = fo.save(x)
    assert np.array_equal(c.q.cpu().numpy(), q) and np.array_equal(c.e.cpu().numpy(), e)
    assert np.array_equal(g.ctx.ckpt8_load(c).cpu().numpy().astype(np.float64), fo.load(q, e, 65536))
    g.close()


@pytest.mark.parametrize("B,K,O", [(3, 24, 65536), (3, 65536, 24)])
def test_widest_layers(B, K, O):
    l = Layer(1, B, K, O)
    c = l.ctx.ckpt8_empty((1, B, O))
    y = torch.empty((1, B, O), device="cuda")
    l.ctx.fp8_linear_forward(l.x8, l.w8, b_off=l.b_off, relu=True, out=y, ckpt=c)
    ref, scale = l.forward(True)
    agree(y.cpu().numpy(), ref, scale)
    s = l.ctx.ckpt8_save(y)
    assert torch.equal(c.q, s.q) and torch.equal(c.e, s.e)
    dy = l.rng.standard_normal((1, B, O)).astype(np.float32)
    dx = torch.empty((1, B, K), device="cuda")
    l.ctx.fp8_linear_backward(l.x8, l.w8, torch.from_numpy(dy).cuda(), w_off=0, b_off=l.b_off, gate=c.q, dx=dx)
    ref, scale = fo.backward(l.xv[0], l.wv[0], dy[0], c.q[0].cpu().numpy())
    agree(l.g.G[0, :O * K].view(O, K).cpu().numpy(), ref[0], scale[0])
    agree(l.g.G[0, l.b_off:l.b_off + O].cpu().numpy(), ref[1], scale[1])
    agree(dx[0].cpu().numpy(), ref[2], scale[2])
    l.close()


def test_most_rows():
    """2^20 rows of a node; the sums over them are formed in 64 bits from the values that the rows stand for."""
    B, K, O = 1 << 20, 20, 12
    X = np.random.default_rng(1).standard_normal((1, O * K + O)).astype(np.float32)
    g = GpuRun(1, O * K + O, wl.topology("ring", 1), 0.1, X=X)
    x8 = g.ctx.ckpt8_save(torch.randn(1, B, K, device="cuda"))
    w8 = g.ctx.fp8_weights(0, O, K)
    wv = torch.from_numpy(fo.weight_values(*fo.weights(X[0, :O * K].reshape(O, K)), K)).cuda()
    xv = g.ctx.ckpt8_load(x8)[0].double()
    y = g.ctx.fp8_linear_forward(x8, w8, b_off=O * K)[0].double()
    ref = xv @ wv.T + torch.from_numpy(X[0, O * K:]).cuda().double()
    assert float((y - ref).abs().max()) <= TOL_SUM * float((xv.abs() @ wv.abs().T).max())
    dy = torch.randn(1, B, O, device="cuda")
    d8 = g.ctx.ckpt8_load(g.ctx.ckpt8_save(dy))[0].double()
    dx = torch.empty(1, B, K, device="cuda")
    g.ctx.fp8_linear_backward(x8, w8, dy, w_off=0, b_off=O * K, dx=dx)
    assert float((dx[0].double() - d8 @ wv).abs().max()) <= TOL_SUM * float((d8.abs() @ wv.abs()).max())
    G = g.G[0].double()
    gw, gb = G[:O * K].view(O, K), G[O * K:O * K + O]
    # 4096 accumulators of 256 samples, added one after the other in fp32: 2^-24 of the partial sum each
    S = d8.abs().T @ xv.abs()
    assert bool(((gw - d8.T @ xv).abs() <= (4096 * 2.0 ** -24 + TOL_SUM) * S).all())
    assert float((gw - d8.T @ xv).norm() / (d8.T @ xv).norm()) <= 1e-4
    # a lane adds 8 rows, 16 warps, then 8192 chunks, each rounding once
    assert bool(((gb - dy[0].double().sum(0)).abs() <= (8192 + 24) * 2.0 ** -24 * dy[0].double().abs().sum(0)).all())
    g.close()


def test_rows_beyond_32_bit_offsets():
    """4.3e9 elements: the last rows lie beyond 2^32 of q and 2^33 bytes of x."""
    torch.cuda.empty_cache()
    R, d = 66000, 65536
    g = GpuRun(1, 32, wl.topology("ring", 1), 0.1)
    x = torch.zeros(R, d, dtype=torch.bfloat16, device="cuda")
    x[-2:] = torch.randn(2, d, device="cuda").bfloat16()
    x[0] = torch.randn(d, device="cuda").bfloat16()
    c = g.ctx.ckpt8_save(x)
    at = [0, R - 2, R - 1]
    q, e = fo.save(x[at].float().cpu().numpy())
    assert np.array_equal(c.q[at].cpu().numpy(), q) and np.array_equal(c.e[at].cpu().numpy(), e)
    assert not c.q[1:R - 2].any()
    x.fill_(7.0)
    g.ctx.ckpt8_load(c, out=x)
    assert np.array_equal(x[at].float().cpu().numpy().astype(np.float64), fo.load(q, e, d)) and not x[1:R - 2].any()
    g.ctx.sync()
    g.close()
    del x, c
    torch.cuda.empty_cache()


def test_layers_beyond_32_bit_offsets():
    """17 nodes of 16384 x 16384: 4.6e9 weights, 18 GB of gradient; the last node's ends against the oracle."""
    torch.cuda.empty_cache()
    n, B, K, O = 17, 2, 16384, 16384
    N = O * K + O
    X = torch.empty(n, N, device="cuda").normal_() * 0.01
    X1, G = torch.empty_like(X), torch.full_like(X, 3.0)
    ctx = binding.Dpsgd(n, N, *wl.ring(n), gamma=0.1)
    ctx.bind(X, X1, G)
    x, dy = torch.randn(n, B, K, device="cuda"), torch.randn(n, B, O, device="cuda")
    x8, w8 = ctx.ckpt8_save(x), ctx.fp8_weights(0, O, K)
    y = ctx.fp8_linear_forward(x8, w8, b_off=O * K)
    dx = torch.empty(n, B, K, device="cuda")
    ctx.fp8_linear_backward(x8, w8, dy, w_off=0, b_off=O * K, dx=dx)
    ctx.sync()
    for i in (0, n - 1):
        xv = fo.load(*fo.save(x[i].cpu().numpy()), K)
        d8 = fo.load(*fo.save(dy[i].cpu().numpy()), O)
        for o in (0, O - 128):
            wv = fo.weight_values(*fo.weights(X[i, o * K:(o + 128) * K].view(128, K).cpu().numpy()), K)
            bias = X[i, O * K + o:O * K + o + 128].cpu().numpy().astype(np.float64)
            ref, scale = fo.forward(xv, wv, bias, False)
            agree(y[i, :, o:o + 128].cpu().numpy(), ref, scale)
            got = G[i, o * K:(o + 128) * K].view(128, K).cpu().numpy().astype(np.float64)
            assert (np.abs(got - d8[:, o:o + 128].T @ xv) <= TOL_SUM * (np.abs(d8[:, o:o + 128]).T @ np.abs(xv))).all()
        wc = torch.from_numpy(w8.q[i, :, K - 128:].cpu().numpy()).view(torch.float8_e4m3fn).double().numpy()
        we = 2.0 ** (w8.e[i, :, K // 128 - 1].cpu().numpy().astype(np.float64) - 127)
        wc *= np.repeat(we, 128)[:, None]
        agree(dx[i, :, K - 128:].cpu().numpy(), d8 @ wc, np.abs(d8) @ np.abs(wc))
        assert np.allclose(G[i, O * K:].cpu().numpy(), dy[i].sum(0).cpu().numpy(), rtol=1e-6, atol=1e-6)
    ctx.close()
    del X, X1, G, x8, w8, y, dx
    torch.cuda.empty_cache()

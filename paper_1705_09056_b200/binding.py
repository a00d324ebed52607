"""Thin ctypes binding of libdpsgd.so: argument marshalling only.

Every step of the D-PSGD iteration (Algorithm 1 of arXiv 1705.09056) runs inside the CUDA
library; torch is used here for device memory and the current stream.  There is no CPU
fallback: if the library is missing or a call fails, a DpsgdError is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdpsgd.so")

OK, ERR_ARG, ERR_W_INVALID, ERR_ALIGN, ERR_STATE, ERR_UNSUPPORTED, ERR_CUDA, ERR_TIMEOUT = range(8)
STATUS_NAMES = ["OK", "ERR_ARG", "ERR_W_INVALID", "ERR_ALIGN", "ERR_STATE", "ERR_UNSUPPORTED",
                "ERR_CUDA", "ERR_TIMEOUT"]
MODEL_LSQ, MODEL_LOGISTIC, MODEL_MLP = 0, 1, 2
MIX_RING, MIX_UNIFORM_DENSE, MIX_TILED_CSR, MIX_GATHER_CSR = 0, 1, 2, 3
DTYPES = {torch.float32: 0, torch.bfloat16: 1}     # DPSGD_F32, DPSGD_BF16
MIX_NAMES = {0: "ring", 1: "uniform_dense", 2: "tiled_csr", 3: "gather_csr"}

_vp, _i32, _i64, _u64, _f32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64,
                               ctypes.c_float)

# name -> argument types (all return int32 status except dpsgd_last_error)
SIGNATURES = {
    "dpsgd_create": [ctypes.POINTER(_vp), _i32, _i64, _vp, _vp, _vp, _f32, _u64],
    "dpsgd_destroy": [_vp],
    "dpsgd_bind": [_vp, _vp, _vp, _vp, _i64, _vp],
    "dpsgd_set_model": [_vp, _i32, _vp, _i32, _f32, _i32, _i32],
    "dpsgd_set_data": [_vp, _vp, _vp, _i64, _i32],
    "dpsgd_sample": [_vp, _u64, _vp],
    "dpsgd_grad": [_vp, _u64],
    "dpsgd_mix_update": [_vp],
    "dpsgd_step": [_vp, _u64],
    "dpsgd_run": [_vp, _u64, _i64],
    "dpsgd_local_step": [_vp, _u64],
    "dpsgd_local_step_nodes": [_vp, _u64, _vp],
    "dpsgd_set_node_batches": [_vp, _vp],
    "dpsgd_set_order": [_vp, _i32],
    "dpsgd_set_fused_step": [_vp, _i32],
    "dpsgd_set_momentum": [_vp, _f32, _vp],
    "dpsgd_mix_update_consensus": [_vp, _vp],
    "dpsgd_step_consensus": [_vp, _u64, _vp],
    "dpsgd_consensus_dist": [_vp, ctypes.POINTER(ctypes.c_double)],
    "dpsgd_sync": [_vp],
    "dpsgd_selftest_wait": [_vp, ctypes.c_uint32],
    "dpsgd_average": [_vp, _vp],
    "dpsgd_conv3x3_forward": [_vp, _vp, _i32, _i32, _i32, _i32, _i32, _i32, _i64, _i64, _i32, _vp],
    "dpsgd_conv3x3_backward": [_vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _i32, _i64, _i64, _i32, _vp],
    "dpsgd_ckpt8_save": [_vp, _vp, _i32, _i64, _i64, _i32, _vp, _vp],
    "dpsgd_ckpt8_load": [_vp, _vp, _vp, _i64, _i32, _vp, _i32, _i64],
    "dpsgd_fp8_weights": [_vp, _i64, _i32, _i32, _vp, _vp],
    "dpsgd_fp8_linear_forward": [_vp, _vp, _vp, _i32, _i32, _i32, _vp, _vp, _i64, _i32, _vp, _i32, _vp, _vp],
    "dpsgd_fp8_linear_backward": [_vp, _vp, _vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _i32, _i64, _i64, _vp, _i32],
    "dpsgd_fp8_reserve": [_vp, _i32, _i32, _i32],
    "dpsgd_mix_update_host": [_vp, _vp, _i64, ctypes.POINTER(ctypes.c_double)],
    "dpsgd_consensus_dist_noalloc": [_vp, _i32, _i64, _i64, _vp, _vp],
    "dpsgd_current": [_vp, ctypes.POINTER(_vp)],
    "dpsgd_set_gamma": [_vp, _f32],
    "dpsgd_mix_kind": [_vp, _i32, ctypes.POINTER(_i32)],
    "dpsgd_launch_count": [_vp, ctypes.POINTER(_i64)],
    "dpsgd_last_error": [_vp],
}

_lib = None


class DpsgdError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES[status] if 0 <= status < 8 else status}: {message}")
        self.status = status


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Loads libdpsgd.so (built in-tree by `python -m paper_1705_09056_b200.build`)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise DpsgdError(ERR_STATE, f"{p} not found: build it with paper_1705_09056_b200/build.py "
                                    "(there is no CPU fallback)")
    lib = ctypes.CDLL(p)
    for name, argtypes in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.argtypes = argtypes
        fn.restype = ctypes.c_char_p if name == "dpsgd_last_error" else ctypes.c_int32
    if path is None:
        _lib = lib
    return lib


def _ptr(t) -> int:
    if t is None:
        return 0
    if isinstance(t, torch.Tensor):
        return t.data_ptr()
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return int(t)


NOALLOC_MAX_LD = 67108864


def _form8(q: torch.Tensor, e: torch.Tensor, d: int):
    assert q.is_cuda and e.is_cuda and q.dtype == torch.uint8 and e.dtype == torch.uint8
    assert q.is_contiguous() and e.is_contiguous()
    assert d >= 1 and q.shape[-1] == -(-d // 16) * 16 and e.shape[-1] == -(-d // 512) * 4


class Ckpt8:
    """Rows in 8 bits: E4M3 bytes q [..., d rounded up to 16], exponent bytes e [..., 4 * ceil(d / 512)] (one per 128
    elements of a row), standing for q * 2^(e - 127).  Checked once, when it is made; do not resize the tensors after."""
    __slots__ = ("q", "e", "d", "lead", "rows")

    def __init__(self, q: torch.Tensor, e: torch.Tensor, d: int):
        _form8(q, e, d)
        assert q.shape[:-1] == e.shape[:-1]
        self.q, self.e, self.d = q, e, d
        self.lead = tuple(q.shape[:-1])
        self.rows = q.numel() // q.shape[-1]


class Fp8Weights:
    """The nodes' weights in 8 bits: q [n][d_out][d_in rounded up to 16], e [n][ceil(d_out / 128)][4 * ceil(d_in / 512)]
    (one exponent per 128 outputs x 128 inputs).  Checked once, when it is made; do not resize the tensors after."""
    __slots__ = ("q", "e", "n", "d_out", "d_in")

    def __init__(self, q: torch.Tensor, e: torch.Tensor, d_in: int):
        _form8(q, e, d_in)
        assert q.dim() == 3 and e.dim() == 3
        self.q, self.e, self.d_in = q, e, d_in
        self.n, self.d_out = q.shape[0], q.shape[1]
        assert e.shape[0] == self.n and e.shape[1] == -(-self.d_out // 128)


def _row_stride(t: torch.Tensor) -> int:
    """Elements between the rows of t [..., d]; the leading dimensions must collapse into one row index."""
    assert t.dim() >= 1 and (t.shape[-1] == 1 or t.stride(-1) == 1), "the last dimension must be contiguous"
    ld, rows = None, 1
    for size, stride in reversed(list(zip(t.shape[:-1], t.stride()[:-1]))):
        if size != 1:
            assert ld is None or stride == ld * rows, "rows must be evenly spaced"
            if ld is None:
                ld = stride
            rows *= size
    return t.shape[-1] if ld is None else ld


def consensus_dist_noalloc(X: torch.Tensor, N: int, out: torch.Tensor, stream=None) -> torch.Tensor:
    """sum_i ||xbar - x_i||^2 of the rows of X (n x ld, columns [N, ld) zero) into the one-element
    float64 CUDA tensor `out`, without any allocation inside the library: for callers that own
    all device memory themselves or have no context.  Asynchronous on the stream; see
    dpsgd_consensus_dist_noalloc in include/dpsgd.h for the size limit and the shared scratch."""
    lib = load_library()
    assert X.is_cuda and X.dtype == torch.float32 and X.is_contiguous() and X.dim() == 2
    assert out.is_cuda and out.dtype == torch.float64 and out.numel() == 1
    s = stream if stream is not None else torch.cuda.current_stream(X.device)
    with torch.cuda.device(X.device):
        st = lib.dpsgd_consensus_dist_noalloc(_ptr(X), X.shape[0], N, X.shape[1], s.cuda_stream, _ptr(out))
    if st != OK:
        raise DpsgdError(st, lib.dpsgd_last_error(None).decode())
    return out


class Dpsgd:
    """One D-PSGD context: n nodes with N parameters each, mixing matrix W (host CSR)."""

    def __init__(self, n: int, N: int, row_ptr, col_idx, val, gamma: float, seed: int = 0):
        self._lib = load_library()
        self._h = _vp()
        rp = np.ascontiguousarray(row_ptr, dtype=np.int32)
        ci = np.ascontiguousarray(col_idx, dtype=np.int32)
        va = np.ascontiguousarray(val, dtype=np.float32)
        st = self._lib.dpsgd_create(ctypes.byref(self._h), n, N, rp.ctypes.data, ci.ctypes.data,
                                    va.ctypes.data, gamma, seed)
        if st != OK:
            msg = self._lib.dpsgd_last_error(None).decode()
            self._h = _vp()
            raise DpsgdError(st, msg)
        self.n, self.N, self.gamma, self.seed = n, N, gamma, seed
        self._keep = []       # tensors bound to the context stay referenced here
        self._data_keep = []

    # -- plumbing --------------------------------------------------------------------------
    def _check(self, st: int):
        if st != OK:
            raise DpsgdError(st, self._lib.dpsgd_last_error(self._h).decode())

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.dpsgd_destroy(self._h)
            self._h = _vp()
        self._keep, self._data_keep = [], []

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the C ABI, one method per entry point --------------------------------------------
    def bind(self, X0: torch.Tensor, X1: torch.Tensor, G: torch.Tensor, stream=None):
        for t in (X0, X1, G):
            assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.dim() == 2
            assert t.shape == X0.shape
        s = stream if stream is not None else torch.cuda.current_stream(X0.device)
        self._check(self._lib.dpsgd_bind(self._h, _ptr(X0), _ptr(X1), _ptr(G), X0.shape[1],
                                         s.cuda_stream))
        self._keep = [X0, X1, G, s]
        self.ld = X0.shape[1]

    def bind_raw(self, X0: int, X1: int, G: int, ld: int, stream: int = 0):
        """Binds raw addresses (for argument-checking tests)."""
        self._check(self._lib.dpsgd_bind(self._h, X0, X1, G, ld, stream))

    def set_model(self, kind: int, dims: Sequence[int], l2_lambda: float = 0.0, batch: int = 1,
                  mlp_precision: int = 0):
        d = np.ascontiguousarray(dims, dtype=np.int32)
        self._check(self._lib.dpsgd_set_model(self._h, kind, d.ctypes.data, len(d), l2_lambda, batch,
                                              mlp_precision))
        self.batch = batch

    def set_data(self, A: torch.Tensor, y: torch.Tensor):
        assert A.is_cuda and A.dtype == torch.float32 and A.is_contiguous() and A.dim() == 3
        assert y.is_cuda and y.is_contiguous() and y.dtype in (torch.float32, torch.int32)
        assert y.shape == A.shape[:2] and A.shape[0] == self.n
        self._check(self._lib.dpsgd_set_data(self._h, _ptr(A), _ptr(y), A.shape[1], A.shape[2]))
        self._data_keep = [A, y]

    def sample(self, k: int, idx: Optional[torch.Tensor] = None) -> torch.Tensor:
        if idx is None:
            idx = torch.empty((self.n, self.batch), dtype=torch.int32, device=self._data_keep[0].device)
        self._check(self._lib.dpsgd_sample(self._h, k, _ptr(idx)))
        return idx

    def grad(self, k: int):
        self._check(self._lib.dpsgd_grad(self._h, k))

    def mix_update(self):
        self._check(self._lib.dpsgd_mix_update(self._h))

    def step(self, k: int):
        self._check(self._lib.dpsgd_step(self._h, k))

    def local_step(self, k: int):
        """Gradient step without communication (several minibatches between exchanges)."""
        self._check(self._lib.dpsgd_local_step(self._h, k))

    def local_step_nodes(self, k: int, active):
        """The local step for the nodes with a non-zero entry of `active` (length n) only."""
        arr = (ctypes.c_int32 * self.n)(*[1 if a else 0 for a in active])
        self._check(self._lib.dpsgd_local_step_nodes(self._h, k, arr))

    def set_node_batches(self, sizes):
        """Per-node minibatch sizes B_i <= batch (length n), or None for the common size."""
        if sizes is None:
            self._check(self._lib.dpsgd_set_node_batches(self._h, None))
            return
        arr = (ctypes.c_int32 * self.n)(*[int(b) for b in sizes])
        self._check(self._lib.dpsgd_set_node_batches(self._h, arr))

    def set_order(self, update_then_mix: bool):
        """Footnote c of Algorithm 1: apply the local gradient first, then average."""
        self._check(self._lib.dpsgd_set_order(self._h, 1 if update_then_mix else 0))

    def set_fused_step(self, mode: int):
        """MLP: let step() apply the gossip step inside the weight-gradient kernels (those blocks of G
        are then not written).  0 off, 1 where it is faster, 2 wherever the kernel applies."""
        self._check(self._lib.dpsgd_set_fused_step(self._h, int(mode)))

    def set_momentum(self, beta: float, V: Optional[torch.Tensor]):
        """Heavy-ball momentum (Section 5.3): V is an n x ld fp32 CUDA tensor, zero at the start; None = off."""
        if V is not None:
            assert V.is_cuda and V.dtype == torch.float32 and V.is_contiguous() and V.shape == self._keep[0].shape
        self._check(self._lib.dpsgd_set_momentum(self._h, beta, _ptr(V)))
        self._momentum_keep = V

    def mix_update_consensus(self, out: torch.Tensor):
        """Gossip step that also writes the new consensus distance into `out` (one float64 on the device)."""
        assert out.is_cuda and out.dtype == torch.float64 and out.numel() >= 1
        self._check(self._lib.dpsgd_mix_update_consensus(self._h, _ptr(out)))

    def step_consensus(self, k: int, out: torch.Tensor):
        assert out.is_cuda and out.dtype == torch.float64 and out.numel() >= 1
        self._check(self._lib.dpsgd_step_consensus(self._h, k, _ptr(out)))

    def run(self, k_first: int, iterations: int):
        """Iterations k_first .. k_first + iterations - 1 of Algorithm 1, enqueued by one call."""
        self._check(self._lib.dpsgd_run(self._h, k_first, iterations))

    def consensus_dist(self) -> float:
        out = ctypes.c_double()
        self._check(self._lib.dpsgd_consensus_dist(self._h, ctypes.byref(out)))
        return out.value

    def sync(self):
        """Waits for the bound stream; raises ERR_TIMEOUT if a kernel's bounded wait ran out meanwhile."""
        self._check(self._lib.dpsgd_sync(self._h))

    def selftest_wait(self, max_polls: int = 4096):
        """Enqueues the self-test CTA whose wait runs out (see dpsgd_selftest_wait)."""
        self._check(self._lib.dpsgd_selftest_wait(self._h, max_polls))

    def conv3x3_forward(self, x: torch.Tensor, c_out: int, stride: int, w_off: int, b_off: int, relu: bool = True,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """3x3 convolution (padding 1) of x [n][B][C][H][W] with every node's own filters, read from the
        current X at columns w_off (filters) and b_off (biases)."""
        assert x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 5 and x.shape[0] == self.n
        _, B, C, H, W = x.shape
        ho, wo = (H - 1) // stride + 1, (W - 1) // stride + 1
        if out is None:
            out = torch.empty((self.n, B, c_out, ho, wo), dtype=torch.float32, device=x.device)
        assert out.is_cuda and out.is_contiguous() and tuple(out.shape) == (self.n, B, c_out, ho, wo)
        self._check(self._lib.dpsgd_conv3x3_forward(self._h, _ptr(x), B, C, H, W, c_out, stride, w_off, b_off,
                                                    1 if relu else 0, _ptr(out)))
        return out

    def conv3x3_backward(self, x: torch.Tensor, y: Optional[torch.Tensor], dy: torch.Tensor, stride: int, w_off: int,
                         b_off: int, relu: bool = True, want_dx: bool = True) -> Optional[torch.Tensor]:
        """Backward of conv3x3_forward: filter and bias gradients (sums over the minibatch) into the bound G at
        columns w_off / b_off; returns the gradient at the layer's input (None when want_dx is False)."""
        assert x.is_cuda and x.is_contiguous() and dy.is_cuda and dy.is_contiguous() and x.dim() == 5 and dy.dim() == 5
        _, B, C, H, W = x.shape
        c_out = dy.shape[2]
        dx = torch.empty_like(x) if want_dx else None
        self._check(self._lib.dpsgd_conv3x3_backward(self._h, _ptr(x), _ptr(y), _ptr(dy), B, C, H, W, c_out, stride,
                                                     w_off, b_off, 1 if relu else 0, _ptr(dx)))
        return dx

    # -- 8-bit layers ----------------------------------------------------------------------
    def ckpt8_empty(self, shape) -> Ckpt8:
        """Uninitialised buffers for the checkpoint of rows of this shape."""
        dev, lead, d = self._keep[0].device, tuple(shape[:-1]), int(shape[-1])
        return Ckpt8(torch.empty(lead + (-(-d // 16) * 16,), dtype=torch.uint8, device=dev),
                     torch.empty(lead + (-(-d // 512) * 4,), dtype=torch.uint8, device=dev), d)

    def fp8_weights_empty(self, d_out: int, d_in: int) -> Fp8Weights:
        dev = self._keep[0].device
        return Fp8Weights(torch.empty((self.n, d_out, -(-d_in // 16) * 16), dtype=torch.uint8, device=dev),
                          torch.empty((self.n, -(-d_out // 128), -(-d_in // 512) * 4), dtype=torch.uint8, device=dev), d_in)

    def ckpt8_save(self, x: torch.Tensor, out: Optional[Ckpt8] = None) -> Ckpt8:
        """Checkpoint of the rows of x [..., d] (fp32 or bf16; rows evenly spaced, elements of a row contiguous)."""
        if out is None:
            out = self.ckpt8_empty(x.shape)
        d = out.d
        assert x.is_cuda and x.dtype in DTYPES and x.shape == out.lead + (d,)
        ld = d if x.is_contiguous() else _row_stride(x)
        self._check(self._lib.dpsgd_ckpt8_save(self._h, x.data_ptr(), DTYPES[x.dtype], ld, out.rows, d, out.q.data_ptr(),
                                               out.e.data_ptr()))
        return out

    def ckpt8_load(self, c: Ckpt8, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The values a checkpoint stands for, as `dtype` (or the type of `out`)."""
        d = c.d
        if out is None:
            out = torch.empty(c.lead + (d,), dtype=dtype, device=c.q.device)
        assert out.is_cuda and out.dtype in DTYPES and out.shape == c.lead + (d,)
        ld = d if out.is_contiguous() else _row_stride(out)
        self._check(self._lib.dpsgd_ckpt8_load(self._h, c.q.data_ptr(), c.e.data_ptr(), c.rows, d, out.data_ptr(),
                                               DTYPES[out.dtype], ld))
        return out

    def fp8_weights(self, w_off: int, d_out: int, d_in: int, out: Optional[Fp8Weights] = None) -> Fp8Weights:
        """8-bit form of every node's d_out x d_in weight block at column w_off of the current X (for other parameters, such
        as the average of the nodes: a context of one node bound to them)."""
        if out is None:
            out = self.fp8_weights_empty(d_out, d_in)
        assert out.n == self.n and out.d_out == d_out and out.d_in == d_in
        self._check(self._lib.dpsgd_fp8_weights(self._h, w_off, d_out, d_in, out.q.data_ptr(), out.e.data_ptr()))
        return out

    def _layer8(self, x: Ckpt8, w: Fp8Weights) -> int:
        assert x.d == w.d_in and w.n == self.n and len(x.lead) == 2 and x.lead[0] == self.n
        return x.lead[1]

    def fp8_linear_forward(self, x: Ckpt8, w: Fp8Weights, b_off: int = -1, relu: bool = False,
                           out: Optional[torch.Tensor] = None, ckpt: Optional[Ckpt8] = None,
                           dtype: torch.dtype = torch.float32) -> Optional[torch.Tensor]:
        """act(x W^T + bias) for every node, x [n][B][d_in] in 8 bits, bias at column b_off of X (-1: none).  Writes the
        output as a checkpoint into `ckpt` when given, and returns it as values in `out` (a new tensor of `dtype` when
        neither is given; None when only the checkpoint is wanted)."""
        batch, d_out = self._layer8(x, w), w.d_out
        y = dt = yq = ye = 0
        if out is None and ckpt is None:
            out = torch.empty((self.n, batch, d_out), dtype=dtype, device=x.q.device)
        if out is not None:
            assert out.is_cuda and out.dtype in DTYPES and out.is_contiguous() and out.shape == (self.n, batch, d_out)
            y, dt = out.data_ptr(), DTYPES[out.dtype]
        if ckpt is not None:
            assert ckpt.d == d_out and ckpt.lead == (self.n, batch)
            yq, ye = ckpt.q.data_ptr(), ckpt.e.data_ptr()
        self._check(self._lib.dpsgd_fp8_linear_forward(self._h, x.q.data_ptr(), x.e.data_ptr(), batch, x.d, d_out,
                                                       w.q.data_ptr(), w.e.data_ptr(), b_off, 1 if relu else 0, y, dt, yq, ye))
        return out

    def fp8_linear_backward(self, x: Ckpt8, w: Fp8Weights, dy: torch.Tensor, w_off: int, b_off: int = -1,
                            gate: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """Backward of fp8_linear_forward: weight and bias gradients (sums over the minibatch) into the bound G at columns
        w_off / b_off, the gradient at the layer's input into dx [n][B][d_in] when given.  `gate`: the q bytes of the
        output's checkpoint for a ReLU layer."""
        batch, d_out = self._layer8(x, w), w.d_out
        assert dy.is_cuda and dy.dtype in DTYPES and dy.is_contiguous() and dy.shape == (self.n, batch, d_out)
        gp = xp = xt = 0
        if gate is not None:
            assert gate.is_cuda and gate.dtype == torch.uint8 and gate.is_contiguous()
            assert gate.shape == (self.n, batch, -(-d_out // 16) * 16)
            gp = gate.data_ptr()
        if dx is not None:
            assert dx.is_cuda and dx.dtype in DTYPES and dx.is_contiguous() and dx.shape == (self.n, batch, x.d)
            xp, xt = dx.data_ptr(), DTYPES[dx.dtype]
        self._check(self._lib.dpsgd_fp8_linear_backward(self._h, x.q.data_ptr(), x.e.data_ptr(), batch, x.d, d_out,
                                                        w.q.data_ptr(), w.e.data_ptr(), gp, dy.data_ptr(), DTYPES[dy.dtype],
                                                        w_off, b_off, xp, xt))
        return dx

    def fp8_reserve(self, batch: int, d_in: int, d_out: int) -> None:
        """Workspace of fp8_linear_backward for layers of up to this size: before the first call that must not allocate, and
        before a call is captured in a CUDA graph."""
        self._check(self._lib.dpsgd_fp8_reserve(self._h, batch, d_in, d_out))

    def average(self, xbar: Optional[torch.Tensor] = None) -> torch.Tensor:
        if xbar is None:
            xbar = torch.empty(self.ld, dtype=torch.float32, device=self._keep[0].device)
        self._check(self._lib.dpsgd_average(self._h, _ptr(xbar)))
        return xbar

    def mix_update_host(self, G_host, ld_host: Optional[int] = None) -> float:
        out = ctypes.c_double()
        if ld_host is None:
            ld_host = G_host.shape[1]
        self._check(self._lib.dpsgd_mix_update_host(self._h, _ptr(G_host), ld_host, ctypes.byref(out)))
        return out.value

    def current(self) -> torch.Tensor:
        p = _vp()
        self._check(self._lib.dpsgd_current(self._h, ctypes.byref(p)))
        for t in self._keep[:2]:
            if t.data_ptr() == p.value:
                return t
        raise DpsgdError(ERR_STATE, "current buffer is not one of the bound tensors")

    def set_gamma(self, gamma: float):
        self._check(self._lib.dpsgd_set_gamma(self._h, gamma))
        self.gamma = gamma

    def mix_kind(self, force: int = -1) -> int:
        out = _i32()
        self._check(self._lib.dpsgd_mix_kind(self._h, force, ctypes.byref(out)))
        return out.value

    def launch_count(self) -> int:
        out = _i64()
        self._check(self._lib.dpsgd_launch_count(self._h, ctypes.byref(out)))
        return out.value

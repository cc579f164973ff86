"""4-bit products whose rows do not start on 16 bytes: an odd number of columns in
the tiles' and the split contraction's ends, short contractions, and gradients
of an odd number of outputs, few rows and many."""
import numpy as np
import pytest

import oracle
from _bounds import assert_within
from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _held(rng, M, K):
    import torch
    codes, e = oracle.hold(rng.standard_normal((M, K)) * np.exp2(rng.integers(-2, 3, (M, K // 32)).repeat(32, axis=1)), 4)
    q, s = oracle.mx_pack(codes, e)
    s[:, M:] = 255                       # what lies in the padding rows must not matter
    return torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), oracle.held_values(codes, e, 4)


def _np(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1500, 2048, 32), (1111, 1029, 96), (600, 1540, 2048), (700, 1031, 4128), (2051, 515, 544)])
def test_linear(gpu, M, N, K, dtype):
    import torch
    rng = np.random.default_rng(N)
    (xq, xs, x), (wq, ws, w) = _held(rng, M, K), _held(rng, N, K)
    flat = torch.from_numpy(rng.standard_normal(N + 1).astype(np.float32)).to(TORCH_DT[dtype]).cuda()
    b, gate = flat[1:], torch.randn(2, N, device="cuda").to(flat.dtype)      # (b one element behind 16 bytes)
    res = torch.randn(M, N, device="cuda").to(flat.dtype)
    prod, size = x @ w.T, np.abs(x) @ np.abs(w).T
    # A sum of K exact products over K / 128 instructions and a few joins, then the bias.
    err = 2.0 ** -23 * (K / 128 + 8) * size
    ref = prod + _np(b)
    out = torch.full((M + 1, N), 7.0, dtype=flat.dtype, device="cuda")
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, b, out[:M])
    assert_within(_np(out[:M]), ref, err + 2.0 ** -23 * np.abs(ref) + HALF[dtype] * (np.abs(ref) + err))
    assert (out[M] == 7.0).all()
    off = [0, M // 3, M]
    y = torch.full((M + 1, N), 7.0, dtype=flat.dtype, device="cuda")
    y[:M] = res
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, b, y[:M], gate=gate, resid=y[:M], off=off)
    g = np.repeat(_np(gate), np.diff(off), axis=0)
    want = _np(res) + g * ref
    tol = np.abs(g) * (err + 2.0 ** -22 * np.abs(ref)) + 2.0 ** -23 * np.abs(want)
    assert_within(_np(y[:M]), want, tol + HALF[dtype] * (np.abs(want) + tol))
    assert (y[M] == 7.0).all()


@pytest.mark.parametrize("K", [32, 160, 1056])
@pytest.mark.parametrize("N", [1, 3, 7, 9, 31, 33, 1027])
@pytest.mark.parametrize("M", [1, 17, 70, 600])
def test_backward(gpu, M, N, K):
    import torch
    rng = np.random.default_rng(N + M)
    wq, ws, w = _held(rng, N, K)
    dy = torch.from_numpy(rng.standard_normal((M, N)).astype(np.float32)).bfloat16()
    if M > 1:
        dy[M // 2, :] = float("nan")     # a row's gradient is its own, also past its end
    dx = torch.full((M + 1, K), 7.0, dtype=dy.dtype, device="cuda")
    gpu.avits_mxfp4_linear_backward(dy.cuda(), wq, ws, dx[:M])
    good = np.arange(M) != (M // 2 if M > 1 else -1)
    d = _np(dy)[good]
    ref, err = d @ w, 2.0 ** -23 * (N / 32 + 8) * (np.abs(d) @ np.abs(w))
    assert_within(_np(dx[:M])[good], ref, err + HALF["bf16"] * (np.abs(ref) + err))
    assert torch.isnan(dx[:M][torch.from_numpy(~good).cuda()]).all() and (dx[M] == 7.0).all()


@pytest.mark.parametrize("M,N,K", [(1, 1, 32), (3, 9, 160), (70, 33, 96), (65, 1027, 1056), (600, 260, 2048), (1300, 513, 544)])
def test_backward_in_fp32(gpu, M, N, K):
    """Values over many powers of two, so that all 24 bits of each count, and a row of NaN."""
    import torch
    rng = np.random.default_rng(N * M)
    wq, ws, w = _held(rng, N, K)
    dy = torch.from_numpy((rng.standard_normal((M, N)) * np.exp2(rng.integers(-40, 40, (M, N)))).astype(np.float32))
    if M > 1:
        dy[M // 2, :] = float("nan")
    dx = torch.full((M + 1, K), 7.0, device="cuda")
    gpu.avits_mxfp4_linear_backward(dy.cuda(), wq, ws, dx[:M])
    good = np.arange(M) != (M // 2 if M > 1 else -1)
    d = _np(dy)[good]
    # Exact products of the three parts of a value, 3 N / 32 instructions and a few joins.
    ref, err = d @ w, 2.0 ** -23 * (3 * N / 32 + 8) * (np.abs(d) @ np.abs(w))
    assert_within(_np(dx[:M])[good], ref, err + HALF["f32"] * np.abs(ref))
    assert torch.isnan(dx[:M][torch.from_numpy(~good).cuda()]).all() and (dx[M] == 7.0).all()


def test_backward_of_infinities(gpu):
    """An infinite gradient stays one: its other parts are 0, not NaN."""
    import torch
    K, N = 64, 8
    w = np.ones((N, K))
    codes, e = oracle.hold(w, 4)
    wq, ws = (torch.from_numpy(a).cuda() for a in oracle.mx_pack(codes, e))
    for dt in (torch.float32, torch.bfloat16):
        dy = torch.zeros(3, N, dtype=dt)
        dy[0, 3], dy[1, 5], dy[2, 0], dy[2, 1] = float("inf"), -float("inf"), 1.0, 3.0e38
        dx = torch.empty(3, K, dtype=dt, device="cuda")
        gpu.avits_mxfp4_linear_backward(dy.cuda(), wq, ws, dx)
        assert (dx[0] == float("inf")).all() and (dx[1] == -float("inf")).all() and torch.equal(dx[2].cpu(), dy[2, 1].expand(K))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 40, 5000])
def test_smallest_and_largest_weights_count(gpu, M, dtype):
    """Scales at both ends: held values below the smallest normal number (0.5 x 2^-127) and near the
    largest, against gradients that bring them back into range."""
    import torch
    N, K = 64, 2048
    rng = np.random.default_rng(5)
    codes = rng.integers(0, 256, (N, K // 2)).astype(np.uint8)
    wq = torch.from_numpy(codes).cuda()
    for code, big in ((0, 2.0 ** 110), (1, 2.0 ** 110), (252, 2.0 ** -110)):
        shape = gpu.avits_mxfp4_scale_shape(N, K)
        s = np.full(shape, code, np.uint8)
        c, e = oracle.mx_unpack(codes, s)
        w = oracle.held_values(c, e, 4)
        dy = torch.from_numpy((rng.standard_normal((M, N)) * big).astype(np.float32)).to(TORCH_DT[dtype])
        dx = torch.empty(M, K, dtype=dy.dtype, device="cuda")
        gpu.avits_mxfp4_linear_backward(dy.cuda(), wq, torch.from_numpy(s).cuda(), dx)
        d = _np(dy)
        ref, err = d @ w, 2.0 ** -23 * (3 * N / 32 + 8) * (np.abs(d) @ np.abs(w))
        assert_within(_np(dx), ref, err + HALF[dtype] * (np.abs(ref) + err), code)

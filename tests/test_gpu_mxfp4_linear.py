"""Products with 4-bit weights on the GPU against exact sums of the held
values, element by element.

Products of two held values are exact; a sum of K of them in fp32 over a chain
of K / 128 matrix instructions (each within 2^-23 of the magnitudes it adds) and
a few joins is off by at most 2^-23 (K / 128 + 8) of the sum of magnitudes; the
gradient's bf16 or fp32 products, over chains of N / 32 or N, likewise."""
import numpy as np
import pytest

import oracle
from _bounds import assert_within
from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _held(rng, M, K, spread=3):
    import torch
    x = rng.standard_normal((M, K)) * np.exp2(rng.integers(-spread, spread + 1, (M, K // 32)).repeat(32, axis=1))
    codes, e = oracle.hold(x, 4)
    q, s = oracle.mx_pack(codes, e)
    s[:, M:] = 255                       # what lies in the padding rows must not matter
    return torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), oracle.held_values(codes, e, 4)


def _t(a, dtype):
    import torch
    return torch.from_numpy(np.asarray(a, np.float32)).to(TORCH_DT[dtype])


def _np(t):
    return t.double().cpu().numpy()


SIZES = [(1, 1, 32), (1, 8, 64), (1, 300, 2048), (3, 33, 96), (16, 64, 256), (17, 65, 288), (64, 128, 544), (65, 63, 32),
         (100, 257, 1056), (255, 256, 512), (257, 520, 768), (600, 1000, 160), (513, 771, 2080), (2, 4096, 5120), (40, 2048, 2048),
         (1030, 2056, 320), (300, 1024, 4096), (4099, 2056, 288), (3000, 3001, 1056),
         (900, 771, 8224), (1030, 1032, 4128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear(gpu, M, N, K, dtype):
    import torch
    rng = np.random.default_rng(M + 31 * N + 7 * K)
    xq, xs, x = _held(rng, M, K)
    wq, ws, w = _held(rng, N, K)
    b = _t(rng.standard_normal(N), dtype)
    out = torch.full((M + 1, N), 7.0, dtype=b.dtype, device="cuda")
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, b.cuda(), out[:M])
    prod, size = x @ w.T, np.abs(x) @ np.abs(w).T
    err = 2.0 ** -23 * (K / 128 + 8) * size
    ref = prod + _np(b)
    assert_within(_np(out[:M]), ref, err + 2.0 ** -23 * np.abs(ref) + HALF[dtype] * (np.abs(ref) + err))
    assert (out[M] == 7.0).all()
    # No bias; gate and residual, in place over the residual, one gate for each image.
    B = min(M, 3)
    off = [0] + sorted(rng.integers(0, M + 1, B - 1).tolist()) + [M]
    gate = _t(rng.standard_normal((B, 2, N)), dtype).cuda()
    res = _t(rng.standard_normal((M, N)), dtype)
    o2 = torch.empty(M, N, dtype=b.dtype, device="cuda")
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, o2)
    assert_within(_np(o2), prod, err + HALF[dtype] * (np.abs(prod) + err))
    y = res.cuda()
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, b.cuda(), y, gate=gate[:, 1], resid=y, off=off)
    g = np.repeat(_np(gate[:, 1]), np.diff(off), axis=0)
    want = _np(res) + g * ref
    tol = np.abs(g) * (err + 2.0 ** -22 * np.abs(ref)) + 2.0 ** -23 * np.abs(want)
    assert_within(_np(y), want, tol + HALF[dtype] * (np.abs(want) + tol))
    shared = gate[0, 1].contiguous()
    y2, y3 = res.cuda(), torch.empty_like(y)
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, b.cuda(), y2, gate=shared, resid=y2)
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, b.cuda(), y3, gate=shared, resid=res.cuda(), off=off)
    assert torch.equal(y2, y3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_backward(gpu, M, N, K, dtype):
    import torch
    rng = np.random.default_rng(M + 17 * N + 3 * K)
    wq, ws, w = _held(rng, N, K)
    dy = _t(rng.standard_normal((M, N)), dtype)
    dx = torch.full((M + 1, K), 7.0, dtype=dy.dtype, device="cuda")
    gpu.avits_mxfp4_linear_backward(dy.cuda(), wq, ws, dx[:M])
    d = _np(dy)
    ref, size = d @ w, np.abs(d) @ np.abs(w)
    err = 2.0 ** -23 * ((N / 32 if dtype == "bf16" else N) + 8) * size
    assert_within(_np(dx[:M]), ref, err + HALF[dtype] * (np.abs(ref) + err))
    assert (dx[M] == 7.0).all()


@pytest.mark.parametrize("M", [5, 300])
def test_marked_blocks_reach_their_row_and_column_only(gpu, M):
    """A block of NaN in one row of x, and in one row of W."""
    import torch
    rng = np.random.default_rng(M)
    N, K = 130, 320
    xq, xs, _ = _held(rng, M, K)
    wq, ws, _ = _held(rng, N, K)
    a = torch.empty(M, N, device="cuda")
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, a)
    xs[4, 3, 1], ws[0, 77, 0] = 255, 255
    b = torch.empty(M, N, device="cuda")
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, b)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[3], bad[:, 77] = True, True
    assert torch.isnan(b[bad]).all() and torch.equal(a[~bad], b[~bad])
    dx = torch.empty(M, K, device="cuda")
    gpu.avits_mxfp4_linear_backward(torch.ones(M, N, device="cuda"), wq, ws, dx)
    assert torch.isnan(dx[:, :32]).all() and not torch.isnan(dx[:, 32:]).any()


def test_other_stream_and_repeats(gpu):
    """Work on a stream that is not the current one, and the same bits every time."""
    import torch
    rng = np.random.default_rng(1)
    xq, xs, x = _held(rng, 700, 640)
    wq, ws, w = _held(rng, 900, 640)
    outs = [torch.empty(700, 900, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    ws_bytes = gpu.avits_mxfp4_linear_workspace_bytes(700, 900, 640)
    work = torch.empty(max(ws_bytes, 1), dtype=torch.uint8, device="cuda")
    for o in outs:
        gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, o, workspace=work, stream=st)
    st.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    ref = x @ w.T
    assert np.abs(_np(outs[0]) - ref).max() <= 2.0 ** -7 * np.abs(ref).max()

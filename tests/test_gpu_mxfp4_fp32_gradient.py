"""The fp32 input gradient of 4-bit products over the whole range of fp32: every bit
of a gradient counts, down to the smallest subnormal number, and with long
contractions."""
import numpy as np
import pytest

import oracle
from _bounds import assert_within

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -24


def _weight(rng, N, K, code):
    """A held weight with one scale byte to a row (code [N]), in both forms."""
    import torch
    codes = rng.integers(0, 16, (N, K)).astype(np.uint8)
    q, s = oracle.mx_pack(codes, np.repeat(np.asarray(code)[:, None] - 127, K // 32, axis=1))
    return torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), oracle.held_values(*oracle.mx_unpack(q, s), 4)


def _check(gpu, dy, wq, ws, w, instructions):
    """A sum's chain of instructions, each within 2^-23 of what it adds, and a few joins; then the
    result's rounding (half a step, at least half the smallest number)."""
    import torch
    M, K = dy.shape[0], w.shape[1]
    dx = torch.full((M + 1, K), 7.0, device="cuda")
    gpu.avits_mxfp4_linear_backward(dy.cuda(), wq, ws, dx[:M])
    d = dy.double().numpy()
    ref, err = d @ w, 2.0 ** -23 * (instructions + 9) * (np.abs(d) @ np.abs(w))
    assert_within(dx[:M].double().cpu().numpy(), ref, err + HALF * np.abs(ref))
    assert (dx[M] == 7.0).all()


@pytest.mark.parametrize("low,high", [(-149, -140), (-140, -133), (-133, -126), (-126, -118), (-118, -109), (-112, -100)])
@pytest.mark.parametrize("M,N,K", [(1, 64, 96), (40, 61, 96), (600, 64, 2048), (5000, 61, 96), (16, 1024, 256)])
def test_the_smallest_gradients(gpu, M, N, K, low, high):
    """Magnitudes from 2^low to 2^high, against weights that bring them back to about 1: five
    parts of a value at most, so 5 N / 32 instructions."""
    import torch
    rng = np.random.default_rng(N + M - low)
    wq, ws, w = _weight(rng, N, K, np.full(N, min(127 - (low + high) // 2, 248)))
    dy = torch.from_numpy((rng.choice([-1, 1], (M, N)) * np.exp2(rng.uniform(low, high, (M, N)))).astype(np.float32))
    _check(gpu, dy, wq, ws, w, 5 * N / 32)


@pytest.mark.parametrize("M,N,K", [(3, 64, 96), (40, 333, 160), (2000, 96, 64)])
def test_small_gradients_among_large_ones(gpu, M, N, K):
    """Every other output's weight is large and its gradient tiny, the others' the other way round:
    all products are of one size."""
    import torch
    rng = np.random.default_rng(N * M)
    e = np.where(np.arange(N) % 2 == 0, 115, -115)
    wq, ws, w = _weight(rng, N, K, 127 + e)
    dy = (rng.standard_normal((M, N)) * np.exp2(-e)).astype(np.float32)
    dy[:, 2] = 0.0
    dy = torch.from_numpy(dy)
    _check(gpu, dy, wq, ws, w, 5 * N / 32)
    # A row's result is its own, whatever other rows hold.
    big = dy.clone()
    big[1:] *= 2.0 ** 8
    a, b = (torch.empty(M, K, device="cuda") for _ in range(2))
    gpu.avits_mxfp4_linear_backward(dy.cuda(), wq, ws, a)
    gpu.avits_mxfp4_linear_backward(big.cuda(), wq, ws, b)
    assert torch.equal(a[0], b[0])


@pytest.mark.parametrize("M,N,K", [(2, 4096, 5120), (40, 2048, 2048), (300, 4100, 512), (1741, 2051, 96), (16, 8192, 256)])
def test_long_contractions(gpu, M, N, K):
    """Values over many powers of two, so that all 24 bits of each count: three parts of a
    value, so 3 N / 32 instructions."""
    import torch
    rng = np.random.default_rng(N)
    wq, ws, w = _weight(rng, N, K, rng.integers(120, 130, N))
    dy = torch.from_numpy((rng.standard_normal((M, N)) * np.exp2(rng.integers(-40, 40, (M, N)))).astype(np.float32))
    _check(gpu, dy, wq, ws, w, 3 * N / 32)


def test_a_bad_gradient_beside_tiny_ones(gpu):
    """Infinities and NaN reach their own row only, also where the rows beside them are tiny."""
    import torch
    N, K = 64, 64
    rng = np.random.default_rng(8)
    wq, ws, w = _weight(rng, N, K, np.full(N, 240))
    dy = torch.from_numpy((rng.standard_normal((5, N)) * 2.0 ** -126).astype(np.float32))
    dy[1, 7], dy[3, 9] = float("inf"), float("nan")
    dx = torch.empty(5, K, device="cuda")
    gpu.avits_mxfp4_linear_backward(dy.cuda(), wq, ws, dx)
    good = [0, 2, 4]
    d = dy[good].double().numpy()
    ref, err = d @ w, 2.0 ** -23 * (5 * N / 32 + 9) * (np.abs(d) @ np.abs(w))
    assert_within(dx[good].double().cpu().numpy(), ref, err + HALF * np.abs(ref))
    assert torch.isnan(dx[3]).all() and not torch.isfinite(dx[1].cpu()[torch.from_numpy(w[7] != 0)]).any()

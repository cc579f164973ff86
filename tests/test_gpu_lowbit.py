"""The block-scaled formats on the GPU, code by code against the oracle, and
the GELU's gradient from them."""
import numpy as np
import pytest

import oracle
from _bounds import assert_within
from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step of the storage type, relative


def _values(rng, M, K, dtype, wild=True):
    """Rows whose blocks have very different sizes, with zeros, ties and the
    format's edges among them, exact in the storage type."""
    import torch
    x = rng.standard_normal((M, K))
    if wild:
        x *= np.exp2(rng.integers(-30, 30, (M, K // 32 + 1)).repeat(32, axis=1)[:, :K])
        x[rng.random((M, K)) < 0.05] = 0.0
        edge = np.array([6.0, 7.0, 7.9375, 5.0, 2.5, 0.25, 448.0, 449.0, 464.0, 480.0, 0.0625, -0.0])
        at = rng.random((M, K)) < 0.2
        x[at] = rng.choice(edge, at.sum()) * rng.choice([-1, 1], at.sum())
        if M > 2:
            x[2] = 0.0                                   # a row of nothing
    return torch.from_numpy(x.astype(np.float32)).to(TORCH_DT[dtype])


SIZES = [(1, 32), (3, 64), (7, 96), (8, 512), (33, 544), (65, 1056), (2, 2080)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K", SIZES)
def test_mxfp4_round_trip(gpu, M, K, dtype):
    import torch
    x = _values(np.random.default_rng(M * 1000 + K), M, K, dtype)
    q = torch.full((M + 1, K // 2), 0xA5, dtype=torch.uint8, device="cuda")     # a row behind the last
    s = torch.full((torch.Size(gpu.avits_mxfp4_scale_shape(M, K))), 7, dtype=torch.uint8, device="cuda")
    assert s.numel() == gpu.avits_mxfp4_scale_bytes(M, K)
    gpu.avits_mxfp4_quantize(x.cuda(), q[:M], s)
    codes, e = oracle.hold(x.float().numpy(), 4)
    wq, wsc = oracle.mx_pack(codes, e)
    assert np.array_equal(q[:M].cpu().numpy(), wq)
    sc = s.cpu().numpy()
    assert np.array_equal(sc[:, :M], wsc[:, :M])
    assert (q[M].cpu().numpy() == 0xA5).all()
    out = torch.full((M + 1, K), 3.0, dtype=x.dtype, device="cuda")
    gpu.avits_mxfp4_dequantize(q[:M], s, out[:M])
    want = torch.from_numpy(oracle.held_values(codes, e, 4)).to(x.dtype)
    assert torch.equal(out[:M].cpu(), want) and (out[M] == 3.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D", SIZES + [(1, 1), (5, 31), (4, 33), (9, 1003), (0, 40)])
def test_ckpt8_round_trip(gpu, M, D, dtype):
    import torch
    x = _values(np.random.default_rng(M * 1000 + D), M, D, dtype)
    ns = (D + 31) // 32
    q = torch.full((M + 1, D), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((M + 1, ns), 9, dtype=torch.uint8, device="cuda")
    gpu.avits_ckpt8_pack(x.cuda(), q[:M], s[:M])
    codes, e = oracle.hold(x.float().numpy(), 8)
    assert np.array_equal(q[:M].cpu().numpy(), codes)
    assert np.array_equal(s[:M].cpu().numpy(), oracle.ckpt_scales(e))
    assert (q[M] == 0xA5).all() and (s[M] == 9).all()
    out = torch.full((M + 1, D), 3.0, dtype=x.dtype, device="cuda")
    gpu.avits_ckpt8_unpack(q[:M], s[:M], out[:M])
    want = torch.from_numpy(oracle.held_values(codes, e, 8)).to(x.dtype)
    assert torch.equal(out[:M].cpu(), want) and (out[M] == 3.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_extremes(gpu, dtype):
    """Infinities, NaN, the smallest and the largest values: a marked block
    reads back as NaN, its neighbours are untouched."""
    import torch
    x = np.ones((6, 128))
    x[0, 5], x[1, 40], x[2, 64] = np.inf, np.nan, -np.inf
    x[3, :32], x[3, 32:64] = 2.0 ** -133, 2.0 ** -126
    x[4, :32], x[4, 32:64] = 3.3895313892515355e38, 2.0 ** 127
    x[5] = 0.0
    t = torch.from_numpy(x.astype(np.float32)).to(TORCH_DT[dtype]).cuda()
    q, s = torch.empty(6, 64, dtype=torch.uint8, device="cuda"), torch.empty(2, 8, 2, dtype=torch.uint8, device="cuda")
    gpu.avits_mxfp4_quantize(t, q, s)
    out = torch.empty_like(t)
    gpu.avits_mxfp4_dequantize(q, s, out)
    codes, e = oracle.hold(t.float().cpu().numpy(), 4)
    want = torch.from_numpy(oracle.held_values(codes, e, 4)).to(t.dtype)
    assert torch.equal(torch.nan_to_num(out.cpu(), nan=-7.0), torch.nan_to_num(want, nan=-7.0))
    assert torch.isnan(out).sum() == 96
    q, s = torch.empty(6, 128, dtype=torch.uint8, device="cuda"), torch.empty(6, 4, dtype=torch.uint8, device="cuda")
    gpu.avits_ckpt8_pack(t, q, s)
    gpu.avits_ckpt8_unpack(q, s, out)
    codes, e = oracle.hold(t.float().cpu().numpy(), 8)
    want = torch.from_numpy(oracle.held_values(codes, e, 8)).to(t.dtype)
    assert torch.equal(torch.nan_to_num(out.cpu(), nan=-7.0), torch.nan_to_num(want, nan=-7.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantised_gelu(gpu, dtype):
    """Every value within half a step of the GELU's (a quarter of itself, 0.25
    scales below one scale), or between 6 and 8 scales and held as 6; the slack
    covers the GELU's own few ulp."""
    import torch
    M, K = 37, 288
    x = _values(np.random.default_rng(3), M, K, dtype, wild=False) * 3
    q, s = torch.empty(M, K // 2, dtype=torch.uint8, device="cuda"), torch.empty(5, 40, 2, dtype=torch.uint8, device="cuda")
    gpu.avits_mxfp4_quantize(x.cuda(), q, s, act=gpu.ACT_GELU)
    codes, e = oracle.mx_unpack(q.cpu().numpy(), s.cpu().numpy())
    got, ref = oracle.held_values(codes, e, 4), oracle.gelu_tanh(x.double().numpy())
    top = np.abs(ref).reshape(M, K // 32, 32).max(axis=2)
    assert (np.abs(e + 2 - np.log2(top) + 0.5) <= 0.5 + 1e-5).all()         # floor(log2) but for ulp at a power of two
    scale = np.repeat(2.0 ** e, 32, axis=1)
    a = np.abs(ref)
    half = np.where(a < 2 * scale, 0.25 * scale, np.where(a < 4 * scale, 0.5 * scale, np.where(a < 6 * scale, scale, a - 6 * scale)))
    assert_within(got, ref, half * (1 + 1e-5) + 1e-5 * scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("M,D", [(1, 1), (3, 32), (5, 77), (64, 512), (9, 1003)])
def test_gelu_backward(gpu, M, D, held, dtype):
    import torch
    rng = np.random.default_rng(D)
    m = _values(rng, M, D, dtype, wild=False) * 4
    da = _values(rng, M, D, dtype, wild=False)
    if D > 40:
        m[0, 3], m[0, 4], m[0, 5] = 60.0, -60.0, 0.0
    ref_m = m.double().numpy()
    args = dict(m=m.cuda())
    if held:
        codes, e = oracle.hold(ref_m, 8)
        ref_m = oracle.held_values(codes, e, 8)
        args = dict(m_q8=torch.from_numpy(codes).cuda(), m_s8=torch.from_numpy(oracle.ckpt_scales(e)).cuda())
    dm = torch.full((M + 1, D), 5.0, dtype=m.dtype, device="cuda")
    gpu.avits_gelu_backward(da.cuda(), dm[:M], **args)
    slope = oracle.gelu_slope(ref_m)
    want = da.double().numpy() * slope
    # With s the logistic of 2 u: the exponent's few roundings are u 2^-21 of it, exp2 and the
    # reciprocal 1 ulp each, so s is off by s (1 - s)(u 2^-21 + 2^-23) + s 2^-22, and the second term
    # s (1 - s) 2 x u' (x u' <= 3 u) by that share of itself and a few roundings more.
    u = 0.7978845608 * (ref_m + 0.044715 * ref_m ** 3)
    s = 1 / (1 + np.exp(-np.minimum(2 * u, 700).clip(-700)))
    u = np.abs(u)
    # A logistic below the smallest normal number, 2^-126, is 0 in fp32's reciprocal; with it goes
    # at most 2^-126 (1 + 6 u), u at most 44 there (exp(-88) = 2^-127).
    size = np.exp(-2 * u) * (1 + 6 * u) * (u + 1) * 2.0 ** -21 + s * 2.0 ** -21 + 2.0 ** -126 * (1 + 6 * np.minimum(u, 44))
    tol = np.abs(da.double().numpy()) * size + HALF[dtype] * np.abs(want)
    assert_within(dm[:M].double().cpu().numpy(), want, tol + 1e-38)
    assert (dm[M] == 5.0).all()
    # In place, over the incoming gradient.
    d2 = da.cuda()
    gpu.avits_gelu_backward(d2, d2, **args)
    assert torch.equal(d2, dm[:M])


def test_infinite_activation_has_a_finite_slope(gpu):
    import torch
    m = torch.tensor([[float("inf"), float("-inf"), 3e38, -3e38, 1e19, -1e19, 0.0, 1.0]], device="cuda")
    dm = torch.empty_like(m)
    gpu.avits_gelu_backward(torch.ones_like(m), dm, m=m)
    assert dm[0, :7].tolist() == [1.0, 0.0, 1.0, 0.0, 1.0, 0.0, 0.5]

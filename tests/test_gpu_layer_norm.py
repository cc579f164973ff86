"""avits_layer_norm and its backward on the GPU against the oracle, element by
element within bounds from the arithmetic.

The bounds: a row's sum runs over D / 64 terms in a lane (or fewer) and a tree of
64, so an average is off by at most u (D / 64 + 16) of the average magnitude
(u = 2^-24); the column sums run over at most 64 terms in a row here; each
further operation adds u of its result.  Storing rounds by half a step."""
import numpy as np
import pytest

import oracle
from _bounds import assert_within
from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}
SIZES = [(1, 1), (1, 256), (2, 7), (5, 64), (3, 512), (65, 520), (4, 1003), (33, 1536), (7, 2048), (130, 96), (9, 4096), (3, 4100),
         (2, 8192), (5, 9000)]


def _case(M, D, B, dtype, seed=0):
    import torch
    rng = np.random.default_rng(seed + M * 7919 + D)
    dt = TORCH_DT[dtype]
    t = lambda a: torch.from_numpy(np.asarray(a, np.float32)).to(dt)  # noqa: E731
    x = rng.standard_normal((M, D)) * np.exp2(rng.integers(-3, 4, (M, 1))) + rng.standard_normal((M, 1))
    mod = t(rng.standard_normal((B, 6, D)) * 0.5)
    cut = sorted(rng.integers(0, M + 1, B - 1).tolist())
    return t(x), mod, [0] + cut + [M], t(rng.standard_normal((M, D))), t(rng.standard_normal((M, D)))


def _np(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D", SIZES)
def test_forward(gpu, M, D, dtype):
    import torch
    B = min(4, M)
    x, mod, off, _, _ = _case(M, D, B, dtype)
    mg = mod.cuda()
    h = torch.full((M + 1, D), 7.0, dtype=x.dtype, device="cuda")
    mean, rstd = (torch.full((M + 1,), 7.0, device="cuda") for _ in range(2))
    gpu.avits_layer_norm(x.cuda(), mg[:, 3], mg[:, 4], h[:M], mean[:M], rstd[:M], off=off)
    xr = _np(x)
    ref, mu, rs = oracle.norm_forward(xr, _np(mod[:, 3]), _np(mod[:, 4]), off, 1e-6)
    k = D / 64 + 16
    emu = U * k * np.abs(xr).mean(axis=1)
    dev = np.abs(xr - mu[:, None])
    # The variance: its average's rounding, and the mean's error through each difference.
    var = ((xr - mu[:, None]) ** 2).mean(axis=1)
    ers = rs * (U * (k + 4) * var + 2 * emu * dev.mean(axis=1) + emu ** 2) / (2 * (var + 1e-6)) + 4 * U * rs
    w = np.abs(1 + np.repeat(_np(mod[:, 4]), np.diff(off), axis=0))
    tol = ((emu * rs)[:, None] + dev * ers[:, None] + 4 * U * dev * rs[:, None]) * w + 2 * U * np.abs(ref)
    tol += U * np.abs(np.repeat(_np(mod[:, 3]), np.diff(off), axis=0)) + HALF[dtype] * np.abs(ref)
    assert_within(_np(h[:M]), ref, tol + 1e-30)
    assert_within(_np(mean[:M]), mu, emu + U * np.abs(mu))
    assert_within(_np(rstd[:M]), rs, ers + U * rs)
    assert (h[M] == 7.0).all() and mean[M] == 7.0 and rstd[M] == 7.0
    # In place, without statistics, without modulation, with one vector for all.
    y = x.cuda()
    gpu.avits_layer_norm(y, mg[:, 3], mg[:, 4], y, off=off)
    assert torch.equal(y, h[:M])
    a, b = torch.empty_like(y), torch.empty_like(y)
    zero = torch.zeros(D, dtype=x.dtype, device="cuda")
    gpu.avits_layer_norm(x.cuda(), None, None, a)
    gpu.avits_layer_norm(x.cuda(), zero, zero, b, off=off)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("M,D", SIZES + [(600, 64), (2100, 40)])
def test_backward(gpu, M, D, held, dtype):
    import torch
    B = min(5, M)
    x, mod, off, dh, dres = _case(M, D, B, dtype, seed=1)
    xr = _np(x)
    _, mu, rs = oracle.norm_forward(xr, _np(mod[:, 3]), _np(mod[:, 4]), off, 1e-6)
    mu, rs = mu.astype(np.float32), rs.astype(np.float32)
    rows = dict(x=x.cuda())
    if held:
        codes, e = oracle.hold(xr, 8)
        xr = oracle.held_values(codes, e, 8)
        rows = dict(x_q8=torch.from_numpy(codes).cuda(), x_s8=torch.from_numpy(oracle.ckpt_scales(e)).cuda())
    scale = mod.cuda()[:, 4]
    dx = torch.full((M + 1, D), 7.0, dtype=x.dtype, device="cuda")
    ds, dt = (torch.full((B + 1, D), 7.0, device="cuda") for _ in range(2))
    dm, dr = torch.from_numpy(mu).cuda(), torch.from_numpy(rs).cuda()
    gpu.avits_layer_norm_backward(dh.cuda(), dm, dr, scale, dx[:M], ds[:B], dt[:B], dres=dres.cuda(), off=off, **rows)
    mu, rs = mu.astype(np.float64), rs.astype(np.float64)
    ref, rds, rdt = oracle.norm_backward(_np(dh), xr, mu, rs, _np(mod[:, 4]), off, _np(dres))
    n = (xr - mu[:, None]) * rs[:, None]
    g = _np(dh) * (1 + np.repeat(_np(mod[:, 4]), np.diff(off), axis=0))
    k = D / 64 + 20
    avg = lambda a: np.abs(a).mean(axis=1, keepdims=True)  # noqa: E731
    inner = U * k * (avg(g) + np.abs(n) * avg(g * n)) + 6 * U * (np.abs(g) + avg(g) + np.abs(n) * avg(g * n))
    tol = rs[:, None] * inner + 2 * U * (np.abs(ref) + np.abs(_np(dres))) + HALF[dtype] * np.abs(ref)
    assert_within(_np(dx[:M]), ref, tol + 1e-30)
    for b in range(B):
        r = slice(off[b], off[b + 1])
        assert_within(_np(ds[b]), rds[b], U * 68 * np.abs(_np(dh) * n)[r].sum(axis=0) + 1e-30)
        assert_within(_np(dt[b]), rdt[b], U * 68 * np.abs(_np(dh))[r].sum(axis=0) + 1e-30)
    assert (dx[M] == 7.0).all() and (ds[B] == 7.0).all() and (dt[B] == 7.0).all()
    # Over the incoming gradient, without the sums: the same rows.
    d2 = dh.cuda()
    gpu.avits_layer_norm_backward(d2, dm, dr, scale, d2, dres=dres.cuda(), off=off, **rows)
    assert torch.equal(d2, dx[:M])
    # One shared scale: its gradient is the sum over the images, and no scale is a scale of 0.
    one, two = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    shared = scale[0].contiguous()
    a = torch.empty(M, D, dtype=x.dtype, device="cuda")
    gpu.avits_layer_norm_backward(dh.cuda(), dm, dr, shared, a, one, two, off=off, **rows)
    same = np.repeat(_np(mod[:1, 4]), B, axis=0)
    _, r1, r2 = oracle.norm_backward(_np(dh), xr, mu, rs, same, off)
    assert_within(_np(one), r1.sum(axis=0), U * 84 * np.abs(_np(dh) * n).sum(axis=0) + 1e-30)
    assert_within(_np(two), r2.sum(axis=0), U * 84 * np.abs(_np(dh)).sum(axis=0) + 1e-30)
    b = torch.empty_like(a)
    gpu.avits_layer_norm_backward(dh.cuda(), dm, dr, None, a, one, two, **rows)
    gpu.avits_layer_norm_backward(dh.cuda(), dm, dr, torch.zeros_like(shared), b, ds[0], dt[0], **rows)
    assert torch.equal(a, b) and torch.equal(one, ds[0]) and torch.equal(two, dt[0])


def test_images_without_rows_and_no_rows_at_all(gpu):
    import torch
    D = 128
    x, mod, _, dh, _ = _case(6, D, 4, "bf16")
    ds, dt = torch.full((4, D), 7.0, device="cuda"), torch.full((4, D), 7.0, device="cuda")
    mean, rstd = torch.zeros(6, device="cuda"), torch.ones(6, device="cuda")
    dx = torch.empty(6, D, dtype=x.dtype, device="cuda")
    gpu.avits_layer_norm_backward(dh.cuda(), mean, rstd, mod.cuda()[:, 4], dx, ds, dt, x=x.cuda(), off=[0, 0, 4, 4, 6])
    assert (ds[[0, 2]] == 0).all() and (dt[[0, 2]] == 0).all() and (ds[1] != 0).any() and (dt[3] != 0).any()
    ds.fill_(7.0)
    dt.fill_(7.0)
    e = torch.empty(0, D, dtype=x.dtype, device="cuda")
    gpu.avits_layer_norm_backward(e, mean[:0], rstd[:0], mod.cuda()[:, 4], e, ds, dt, x=e, off=[0, 0, 0, 0, 0])
    assert (ds == 0).all() and (dt == 0).all()
    gpu.avits_layer_norm(e, None, None, e)


@pytest.mark.parametrize("D", [64, 1003, 2048])
def test_a_bad_row_stays_its_own(gpu, D):
    """Infinities and NaN in one row reach that row and the column sums only."""
    import torch
    x, mod, _, dh, _ = _case(9, D, 1, "f32")
    x2 = x.clone()
    x2[4, D // 2] = float("inf")
    x2[7, 0] = float("nan")
    h = [torch.empty(9, D, device="cuda") for _ in range(2)]
    for a, o in zip((x, x2), h):
        gpu.avits_layer_norm(a.cuda(), None, None, o)
    good = [i for i in range(9) if i not in (4, 7)]
    assert torch.equal(h[0][good], h[1][good]) and torch.isnan(h[1][7]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unaligned_rows(gpu, dtype):
    """A slice that starts at any element gives what the aligned tensor gives within rounding."""
    import torch
    D = 256
    x, mod, _, dh, _ = _case(5, D, 1, dtype)
    big = torch.zeros(5 * D + 1, dtype=x.dtype, device="cuda")
    xs = big[1:].view(5, D)
    xs.copy_(x.cuda())
    h, h2 = torch.empty(5, D, dtype=x.dtype, device="cuda"), torch.empty(5, D, dtype=x.dtype, device="cuda")
    m, r, m2, r2 = (torch.empty(5, device="cuda") for _ in range(4))
    gpu.avits_layer_norm(x.cuda(), None, None, h, m, r)
    gpu.avits_layer_norm(xs, None, None, h2, m2, r2)
    # Both are within the same few roundings of the exact rows.
    assert (h.double() - h2.double()).abs().max() <= 2 * HALF[dtype] * h.double().abs().max() + 64 * U
    dx, dx2 = torch.empty_like(h), torch.empty_like(h)
    a = [torch.empty(D, device="cuda") for _ in range(4)]
    gpu.avits_layer_norm_backward(dh.cuda(), m, r, None, dx, a[0], a[1], x=x.cuda())
    gpu.avits_layer_norm_backward(dh.cuda(), m, r, None, dx2, a[2], a[3], x=xs)
    assert (dx.double() - dx2.double()).abs().max() <= 2 * HALF[dtype] * dx.double().abs().max() + 256 * U
    assert (a[0] - a[2]).abs().max() <= 64 * U * 5 * 16 and (a[1] - a[3]).abs().max() <= 64 * U * 5 * 16

"""The modulated layer norm and its backward at widths that do not divide by a
16-byte chunk, off its alignment, in place, and around the sizes where the
kernels' forms change."""
import numpy as np
import pytest

import oracle
from _bounds import assert_within
from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}
WIDTHS = [3, 4, 5, 8, 9, 15, 37, 63, 257, 259, 511, 513, 1021, 1030, 1537, 2049, 2055, 2561, 3585, 4095, 4097, 6001, 8191, 8193]


def _np(t):
    return t.double().cpu().numpy()


def _off_grid(t):
    """The same rows starting one element behind 16 bytes, and that memory."""
    import torch
    flat = torch.full((t.numel() + 17,), 9, dtype=t.dtype, device="cuda")
    rows = flat[1:1 + t.numel()].view(t.shape)
    rows.copy_(t)
    return rows, flat


def _untouched(flat, n):
    return bool((flat[:1] == 9).all() and (flat[1 + n:] == 9).all())


def _case(D, dtype, B=3):
    import torch
    M = 75 if D < 1000 else 21
    rng = np.random.default_rng(D)
    t = lambda a: torch.from_numpy(np.asarray(a, np.float32)).to(TORCH_DT[dtype])  # noqa: E731
    x = t(rng.standard_normal((M, D)) + rng.standard_normal((M, 1)))
    off = [0] + sorted(rng.integers(0, M + 1, B - 1).tolist()) + [M]
    return M, x, t(rng.standard_normal((B, 2, D)) * 0.5), off, t(rng.standard_normal((M, D))), t(rng.standard_normal((M, D)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_forward(gpu, D, dtype):
    import torch
    M, x, mod, off, _, _ = _case(D, dtype)
    mg = mod.cuda()
    xg, _ = _off_grid(x)
    h, hf = _off_grid(torch.empty_like(x))
    mean, mf = _off_grid(torch.empty(M))
    rstd, rf = _off_grid(torch.empty(M))
    gpu.avits_layer_norm(xg, mg[:, 0], mg[:, 1], h, mean, rstd, off=off)
    xr = _np(x)
    ref, mu, rs = oracle.norm_forward(xr, _np(mod[:, 0]), _np(mod[:, 1]), off, 1e-6)
    # A row's sum: D / 64 terms in a lane (or fewer) and a tree of 64; the variance, its average's rounding
    # and the mean's error through each difference; a few operations more.
    k = D / 64 + 16
    emu = U * k * np.abs(xr).mean(axis=1)
    dev = np.abs(xr - mu[:, None])
    var = (dev ** 2).mean(axis=1)
    ers = rs * (U * (k + 4) * var + 2 * emu * dev.mean(axis=1) + emu ** 2) / (2 * (var + 1e-6)) + 4 * U * rs
    w = np.abs(1 + np.repeat(_np(mod[:, 1]), np.diff(off), axis=0))
    tol = ((emu * rs)[:, None] + dev * ers[:, None] + 4 * U * dev * rs[:, None]) * w + 2 * U * np.abs(ref)
    tol += U * np.abs(np.repeat(_np(mod[:, 0]), np.diff(off), axis=0)) + HALF[dtype] * np.abs(ref)
    assert_within(_np(h), ref, tol + 1e-30)
    assert_within(_np(mean), mu, emu + U * np.abs(mu))
    assert_within(_np(rstd), rs, ers)
    assert _untouched(hf, M * D) and _untouched(mf, M) and _untouched(rf, M)
    y, yf = _off_grid(x)
    gpu.avits_layer_norm(y, mg[:, 0], mg[:, 1], y, off=off)
    assert torch.equal(y, h) and _untouched(yf, M * D)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("D", WIDTHS)
def test_backward(gpu, D, held, dtype):
    import torch
    M, x, mod, off, dh, dres = _case(D, dtype)
    B = len(off) - 1
    xr = _np(x)
    _, mu, rs = oracle.norm_forward(xr, _np(mod[:, 0]), _np(mod[:, 1]), off, 1e-6)
    mean, rstd = (torch.from_numpy(a.astype(np.float32)).cuda() for a in (mu, rs))
    args = dict(x=_off_grid(x)[0])
    if held:
        codes, e = oracle.hold(xr, 8)
        xr = oracle.held_values(codes, e, 8)
        args = dict(x_q8=_off_grid(torch.from_numpy(codes))[0], x_s8=torch.from_numpy(oracle.ckpt_scales(e)).cuda())
    sc = mod.cuda()[:, 1]
    dx, xf = _off_grid(torch.empty_like(x))
    ds, sf = _off_grid(torch.empty(B, D))
    dt, tf = _off_grid(torch.empty(B, D))
    gpu.avits_layer_norm_backward(_off_grid(dh)[0], mean, rstd, sc, dx, ds, dt, dres=_off_grid(dres)[0], off=off, **args)
    mu, rs, d, r = _np(mean), _np(rstd), _np(dh), _np(dres)
    ref, rds, rdt = oracle.norm_backward(d, xr, mu, rs, _np(mod[:, 1]), off, r)
    n = (xr - mu[:, None]) * rs[:, None]
    w = 1 + np.repeat(_np(mod[:, 1]), np.diff(off), axis=0)
    k = D / 64 + 16
    # n is off by 2 roundings; a row's averages by k of their average magnitudes, and a rounding or two a term.
    en = 3 * U * (np.abs(n) + np.abs(mu * rs)[:, None])
    g = np.abs(d * w)
    ea = U * (k + 2) * g.mean(axis=1)
    eb = U * (k + 4) * (g * np.abs(n)).mean(axis=1) + (g * en).mean(axis=1)
    an = np.abs((d * w * n).mean(axis=1))
    tol = rs[:, None] * (4 * U * g + ea[:, None] + np.abs(n) * eb[:, None] + en * an[:, None] +
                         4 * U * (g.mean(axis=1)[:, None] + np.abs(n) * an[:, None])) + 2 * U * (np.abs(ref) + np.abs(r))
    assert_within(_np(dx), ref, tol + HALF[dtype] * (np.abs(ref) + tol), "dx")
    # The column sums: at most 75 terms of a column, each product a rounding and n's error.
    rows = np.repeat(np.arange(B), np.diff(off))
    size = lambda a: np.stack([a[rows == b].sum(axis=0) for b in range(B)])  # noqa: E731
    assert_within(_np(ds), rds, U * 80 * size(np.abs(d * n)) + size(np.abs(d) * en) + 1e-30, "dscale")
    assert_within(_np(dt), rdt, U * 80 * size(np.abs(d)) + 1e-30, "dshift")
    assert _untouched(xf, M * D) and _untouched(sf, B * D) and _untouched(tf, B * D)
    # In place over either gradient.
    for over in (0, 1):
        a = [_off_grid(dh), _off_grid(dres)]
        gpu.avits_layer_norm_backward(a[0][0], mean, rstd, sc, a[over][0], dres=a[1][0], off=off, **args)
        assert torch.equal(a[over][0], dx) and _untouched(a[over][1], M * D)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [509, 512, 2053])
def test_many_rows(gpu, D, dtype):
    """Column sums over many chunks of rows, images of very different sizes."""
    import torch
    M, B = 9001, 4
    off = [0, 3, 3, 8000, M]
    gen = torch.Generator("cuda").manual_seed(D)
    dh, x = (torch.randn(M, D, device="cuda", generator=gen).to(TORCH_DT[dtype]) for _ in range(2))
    sc = torch.randn(B, D, device="cuda", generator=gen).to(TORCH_DT[dtype])
    mean, rstd = torch.randn(M, device="cuda", generator=gen) * 0.1, torch.rand(M, device="cuda", generator=gen) + 0.5
    dx, ds, dt = torch.empty_like(x), torch.empty(B, D, device="cuda"), torch.empty(B, D, device="cuda")
    gpu.avits_layer_norm_backward(dh, mean, rstd, sc, dx, ds, dt, x=x, off=off)
    d, n = dh.double(), (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    for b in range(B):
        rows = slice(off[b], off[b + 1])
        for got, t in ((ds, d * n), (dt, d)):
            # Chunks of at most 40 rows in order, 64 strands of their sums, a tree: below 128 terms in a row.
            assert_within(_np(got[b]), _np(t[rows].sum(0)), U * 132 * _np(t[rows].abs().sum(0)) + 1e-30, b)
    g = d * (1 + sc.double().repeat_interleave(torch.tensor(np.diff(off)).cuda(), 0))
    ref = rstd.double()[:, None] * (g - g.mean(1, True) - n * (g * n).mean(1, True))
    err = (dx.double() - ref).abs().max() / ref.abs().max()
    assert err < HALF[dtype] + 1e-5


@pytest.mark.parametrize("D", [5, 64, 1003])
@pytest.mark.parametrize("M,B", [(1, 1), (8, 1), (9, 1), (20, 3), (24, 3), (300, 3)])
def test_one_of_the_sums(gpu, M, B, D):
    """dscale or dshift alone, with few rows (whose sums are written at once) and with more: the bits of both."""
    import torch
    gen = torch.Generator("cuda").manual_seed(M + D)
    dh, x = (torch.randn(M, D, device="cuda", generator=gen) for _ in range(2))
    mean, rstd = torch.randn(M, device="cuda", generator=gen), torch.rand(M, device="cuda", generator=gen) + 0.5
    off = [M * i // B for i in range(B + 1)]
    for sc, shape in ((torch.randn(B, D, device="cuda", generator=gen), (B + 1, D)), (torch.randn(D, device="cuda", generator=gen), (2, D))):
        both = [torch.full(shape, 7.0, device="cuda") for _ in range(2)]
        view = lambda t: t[:-1] if sc.dim() == 2 else t[0]  # noqa: E731
        dx = [torch.empty_like(x) for _ in range(4)]
        gpu.avits_layer_norm_backward(dh, mean, rstd, sc, dx[0], view(both[0]), view(both[1]), x=x, off=off)
        one = [torch.full(shape, 7.0, device="cuda") for _ in range(2)]
        gpu.avits_layer_norm_backward(dh, mean, rstd, sc, dx[1], view(one[0]), None, x=x, off=off)
        gpu.avits_layer_norm_backward(dh, mean, rstd, sc, dx[2], None, view(one[1]), x=x, off=off)
        gpu.avits_layer_norm_backward(dh, mean, rstd, sc, dx[3], None, None, x=x, off=off)
        assert torch.equal(both[0], one[0]) and torch.equal(both[1], one[1]) and all(torch.equal(dx[0], d) for d in dx[1:])
        assert (both[0][-1] == 7.0).all() and (both[1][-1] == 7.0).all()
        n = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        for got, t in ((both[0], dh.double() * n), (both[1], dh.double())):
            for i in range(B if sc.dim() == 2 else 1):
                r = slice(off[i], off[i + 1]) if sc.dim() == 2 else slice(0, M)
                assert_within(_np(got[i]), _np(t[r].sum(0)), U * 132 * _np(t[r].abs().sum(0)) + 1e-30)

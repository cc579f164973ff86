"""Infinities and NaN in the training operators and in the quantised GELU: what they
reach and what they leave alone.  And rows that start at any element, bit for bit."""
import numpy as np
import pytest

import oracle
from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu


def _rand(seed, *shape):
    import torch
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def _rows(gpu, x, held):
    """The forward's rows as the backward takes them."""
    import torch
    if not held:
        return dict(x=x)
    M, D = x.shape
    q, s = torch.empty(M, D, dtype=torch.uint8, device="cuda"), torch.empty(M, (D + 31) // 32, dtype=torch.uint8, device="cuda")
    gpu.avits_ckpt8_pack(x, q, s)
    return dict(x_q8=q, x_s8=s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("M,D", [(9, 3), (9, 64), (9, 1003), (130, 2048), (131, 2050), (40, 5000), (12, 9001)])
def test_norm_backward(gpu, M, D, held, dtype):
    """A NaN in a row of dh, an infinity in a row of x (whose statistics are NaN then): those rows are
    lost, the other rows and the other images' sums keep their bits."""
    import torch
    dt = TORCH_DT[dtype]
    x, dh, dres = (_rand(i, M, D).to(dt) for i in range(3))
    scale = _rand(3, 3, D).to(dt).cuda()
    off, a, b = [0, M // 3, 2 * M // 3, M], 1, M // 3 + 1       # one bad row in each of the first two images

    def run(x, dh):
        x = x.cuda()
        h = torch.empty_like(x)
        mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        gpu.avits_layer_norm(x, None, None, h, mean, rstd)
        dx = torch.empty_like(x)
        ds, dt_ = torch.empty(3, D, device="cuda"), torch.empty(3, D, device="cuda")
        gpu.avits_layer_norm_backward(dh.cuda(), mean, rstd, scale, dx, ds, dt_, dres=dres.cuda(), off=off, **_rows(gpu, x, held))
        return dx, ds, dt_

    good = run(x, dh)
    x2, dh2 = x.clone(), dh.clone()
    dh2[a, D // 2] = float("nan")
    x2[b, D - 1] = float("inf")
    dx, ds, dt_ = run(x2, dh2)
    rest = [i for i in range(M) if i not in (a, b)]
    assert torch.equal(dx[rest], good[0][rest])
    assert torch.isnan(dx[a]).all() and torch.isnan(dx[b]).all()
    # dh's NaN is one column's; a row without statistics is in every column of its image's dscale.
    col = torch.arange(D, device="cuda") != D // 2
    assert torch.isnan(ds[0, ~col]).all() and torch.isnan(dt_[0, ~col]).all()
    assert torch.equal(ds[0, col], good[1][0, col]) and torch.equal(dt_[0, col], good[2][0, col])
    assert torch.isnan(ds[1]).all() and torch.equal(dt_[1], good[2][1])
    assert torch.equal(ds[2], good[1][2]) and torch.equal(dt_[2], good[2][2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 1003])
def test_norm_forward_rows_without_statistics(gpu, D, dtype):
    import torch
    x = _rand(1, 6, D).to(TORCH_DT[dtype])
    x[1, 0], x[3, D - 1], x[4, 2] = float("inf"), float("nan"), -float("inf")
    h = torch.empty(6, D, dtype=x.dtype, device="cuda")
    mean, rstd = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    gpu.avits_layer_norm(x.cuda(), None, None, h, mean, rstd)
    bad = torch.tensor([False, True, False, True, True, False])
    assert torch.isnan(h.cpu()[bad]).all() and torch.isnan(rstd.cpu()[bad]).all()
    assert torch.isfinite(h.cpu()[~bad]).all() and mean[1] == float("inf") and mean[4] == -float("inf") and torch.isnan(mean[3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantised_gelu(gpu, dtype):
    """The GELU of minus infinity is 0, so its block is an ordinary one; plus infinity and NaN mark theirs."""
    import torch
    x = _rand(5, 5, 96).to(TORCH_DT[dtype])
    ref = x.clone()
    x[0, 3], ref[0, 3] = -float("inf"), -1e4
    x[1, 40], x[2, 95], x[3, 0] = float("inf"), float("nan"), -3.0e38
    ref[3, 0] = -1e4

    def quantise(t):
        q, s = torch.empty(5, 48, dtype=torch.uint8, device="cuda"), torch.empty(2, 8, 2, dtype=torch.uint8, device="cuda")
        gpu.avits_mxfp4_quantize(t.cuda(), q, s, act=gpu.ACT_GELU)
        out = torch.empty(5, 96, device="cuda")
        gpu.avits_mxfp4_dequantize(q, s, out)
        return out, s

    out, s = quantise(x)
    want, _ = quantise(ref)
    marked = torch.zeros(5, 96, dtype=torch.bool, device="cuda")
    marked[1, 32:64], marked[2, 64:] = True, True
    assert torch.isnan(out[marked]).all() and torch.equal(out[~marked], want[~marked])
    assert s[0, 1, 1] == 255 and s[1, 2, 0] == 255 and out[0, 3] == 0 and out[3, 0] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [96, 45])
def test_gelu_backward(gpu, dtype, D):
    """The slope is 1 at plus infinity, 0 at minus infinity and far below zero, NaN at NaN; from 8 bits a marked
    block is NaN throughout."""
    import torch
    dt = TORCH_DT[dtype]
    m, da = _rand(1, 4, D).to(dt), _rand(2, 4, D).to(dt)
    m[0, 1], m[0, 2], m[0, 3], m[0, 4], m[1, 33] = float("inf"), -float("inf"), 3.0e38, -3.0e38, float("nan")
    dm = torch.empty(4, D, dtype=dt, device="cuda")
    gpu.avits_gelu_backward(da.cuda(), dm, m=m.cuda())
    d = dm.cpu()
    assert d[0, 1] == da[0, 1] and d[0, 2] == 0 and d[0, 3] == da[0, 3] and d[0, 4] == 0 and torch.isnan(d[1, 33])
    assert torch.isnan(d).sum() == 1
    held = _rows(gpu, m.cuda(), True)
    gpu.avits_gelu_backward(da.cuda(), dm, m_q8=held["x_q8"], m_s8=held["x_s8"])
    lost = torch.zeros(4, D, dtype=torch.bool)
    lost[0, :32], lost[1, 32:64] = True, True
    d = dm.cpu()
    assert torch.equal(torch.isnan(d), lost)
    codes, e = oracle.hold(m.double().numpy(), 8)
    v = oracle.held_values(codes, e, 8)
    ref = da.double().numpy() * oracle.gelu_slope(np.where(lost.numpy(), 0.0, v))
    # exp and the reciprocal within 2 ulp each, a few operations, an argument of at most 20 in exp2.
    tol = 2.0 ** -17 * np.abs(da.double().numpy()) + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref)
    assert (np.abs(d.double().numpy() - ref) <= tol)[~lost.numpy()].all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [5, 256, 1003, 5000])
def test_rows_at_any_element(gpu, D, dtype):
    """Tensors that start one element behind 16 bytes, and codes one byte: the aligned ones' bits."""
    import torch
    M, dt = 9, TORCH_DT[dtype]

    def shifted(t):
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        return flat[1:].view(t.shape).copy_(t)

    x, dh, dres = (_rand(i, M, D).to(dt).cuda() for i in range(3))
    shift, scale = (_rand(i, D).to(dt).cuda() for i in (3, 4))

    def run(move):
        h, dx = move(torch.zeros_like(x)), move(torch.zeros_like(x))
        mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        ds, dt_ = (move(torch.zeros(D, device="cuda")) for _ in range(2))
        gpu.avits_layer_norm(move(x), move(shift), move(scale), h, mean, rstd)
        got = [h, mean, rstd]
        for held in (False, True):
            rows = {k: move(v) for k, v in _rows(gpu, x, held).items()}
            gpu.avits_layer_norm_backward(move(dh), mean, rstd, move(scale), dx, ds, dt_, dres=move(dres), **rows)
            got += [t.clone() for t in (dx, ds, dt_)]
        held = _rows(gpu, x, True)
        q, s = move(torch.zeros_like(held["x_q8"])), move(torch.zeros_like(held["x_s8"]))
        gpu.avits_ckpt8_pack(move(x), q, s)
        back, dm = move(torch.zeros_like(x)), move(torch.zeros_like(x))
        gpu.avits_ckpt8_unpack(q, s, back)
        gpu.avits_gelu_backward(move(dh), dm, m_q8=q, m_s8=s)
        plain = move(torch.zeros_like(x))
        gpu.avits_gelu_backward(move(dh), plain, m=move(x))
        return got + [q, s, back, dm, plain]

    a, b = run(lambda t: t), run(shifted)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D", [(20, 96), (700, 2048), (700, 1003)])
def test_norm_of_sixteen_images(gpu, M, D, dtype):
    """Every image's rows and sums as in a call of its own (sums within their order's rounding)."""
    import torch
    dt = TORCH_DT[dtype]
    x, dh = _rand(1, M, D).to(dt).cuda(), _rand(2, M, D).to(dt).cuda()
    mod = _rand(3, 16, 6, D).to(dt).cuda()
    shift, scale = mod[:, 0], mod[:, 1]
    cut = torch.randint(0, M + 1, (15,), generator=torch.Generator().manual_seed(D)).sort().values.tolist()
    off = [0] + cut + [M]
    h, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    ds, dt_ = torch.empty(16, D, device="cuda"), torch.empty(16, D, device="cuda")
    gpu.avits_layer_norm(x, shift, scale, h, mean, rstd, off=off)
    gpu.avits_layer_norm_backward(dh, mean, rstd, scale, dx, ds, dt_, x=x, off=off)
    for i in range(16):
        r = slice(off[i], off[i + 1])
        n = off[i + 1] - off[i]
        one, d1 = torch.empty_like(x[r]), torch.empty_like(x[r])
        s1, t1 = torch.empty(1, D, device="cuda"), torch.empty(1, D, device="cuda")
        gpu.avits_layer_norm(x[r], shift[i:i + 1], scale[i:i + 1], one)
        gpu.avits_layer_norm_backward(dh[r], mean[r], rstd[r], scale[i:i + 1], d1, s1, t1, x=x[r])
        assert torch.equal(h[r], one) and torch.equal(dx[r], d1), i
        # Two orders of n sums of fp32: n 2^-24 of the magnitudes each.
        size = (dh[r].double() * ((x[r].double() - mean[r, None].double()) * rstd[r, None].double())).abs().sum(0)
        assert ((ds[i] - s1[0]).abs().double() <= 2 * (n + 4) * 2.0 ** -24 * size + 1e-30).all()
        assert ((dt_[i] - t1[0]).abs().double() <= 2 * (n + 4) * 2.0 ** -24 * dh[r].double().abs().sum(0) + 1e-30).all()

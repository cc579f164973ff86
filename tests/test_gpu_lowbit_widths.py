"""Rows of any width and alignment through the 8-bit activations and the GELU's
gradient: widths around a group of eight and a block of 32, few rows and many."""
import numpy as np
import pytest

import oracle
from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu

WIDTHS = [1, 2, 7, 8, 9, 15, 16, 31, 33, 36, 39, 40, 41, 63, 65, 71, 100, 259, 513, 517, 545, 1027, 2049, 2055]


def _off_grid(t):
    """The same rows starting one element behind 16 bytes, and that memory with what is around them."""
    import torch
    flat = torch.full((t.numel() + 17,), 9, dtype=t.dtype, device="cuda")
    rows = flat[1:1 + t.numel()].view(t.shape)
    rows.copy_(t)
    return rows, flat


def _untouched(flat, n):
    return bool((flat[:1] == 9).all() and (flat[1 + n:] == 9).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_any_width(gpu, D, dtype):
    import torch
    M, ns = (301 if D < 1000 else 37), (D + 31) // 32
    rng = np.random.default_rng(D)
    x = rng.standard_normal((M, D)) * np.exp2(rng.integers(-20, 20, (M, ns)).repeat(32, axis=1)[:, :D])
    x[M // 2] = 0.0
    x[M // 3, D - 1] = np.inf
    x = torch.from_numpy(x.astype(np.float32)).to(TORCH_DT[dtype])
    codes, e = oracle.hold(x.double().numpy(), 8)
    xg, _ = _off_grid(x)
    q, qf = _off_grid(torch.empty(M, D, dtype=torch.uint8))
    s, sf = _off_grid(torch.empty(M, ns, dtype=torch.uint8))
    gpu.avits_ckpt8_pack(xg, q, s)
    good = np.isfinite(x.float().numpy()).reshape(M, D)
    good[M // 3, (D - 1) // 32 * 32:] = False            # the marked block's codes are not used
    assert np.array_equal(s.cpu().numpy(), oracle.ckpt_scales(e))
    assert np.array_equal(q.cpu().numpy()[good], codes[good])
    out, of = _off_grid(torch.empty_like(x))
    gpu.avits_ckpt8_unpack(q, s, out)
    want = torch.from_numpy(oracle.held_values(codes, e, 8)).to(x.dtype)
    assert torch.equal(torch.nan_to_num(out.cpu(), nan=-7.0), torch.nan_to_num(want, nan=-7.0))
    assert torch.isnan(out).sum() == D - (D - 1) // 32 * 32
    assert _untouched(qf, M * D) and _untouched(sf, M * ns) and _untouched(of, M * D)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_gelu_backward_as_in_whole_blocks(gpu, D, dtype):
    """The bits that rows padded to whole blocks give, whose kernel is another; in place too."""
    import torch
    M, dt = (301 if D < 1000 else 37), TORCH_DT[dtype]
    W = (D + 31) // 32 * 32
    g = torch.Generator("cuda").manual_seed(D)
    da, m = (torch.zeros(M, W, dtype=dt, device="cuda") for _ in range(2))
    for t in (da, m):
        t[:, :D] = torch.randn(M, D, device="cuda", generator=g) * 2
    q, s = torch.empty(M, W, dtype=torch.uint8, device="cuda"), torch.empty(M, W // 32, dtype=torch.uint8, device="cuda")
    gpu.avits_ckpt8_pack(m, q, s)
    for wide, args in ((dict(m=m), dict(m=_off_grid(m[:, :D])[0])), (dict(m_q8=q, m_s8=s), dict(m_q8=_off_grid(q[:, :D])[0], m_s8=s))):
        want = torch.empty_like(m)
        gpu.avits_gelu_backward(da, want, **wide)
        d, flat = _off_grid(da[:, :D])
        dm, df = _off_grid(torch.empty(M, D, dtype=dt))
        gpu.avits_gelu_backward(d, dm, **args)
        assert torch.equal(dm, want[:, :D])
        gpu.avits_gelu_backward(d, d, **args)
        assert torch.equal(d, dm) and _untouched(flat, M * D) and _untouched(df, M * D)


@pytest.mark.parametrize("M,D", [(90001, 37), (9001, 1001), (3, 100003)])
def test_many_rows_and_long_ones(gpu, M, D):
    import torch
    x = torch.randn(M, D, device="cuda", generator=torch.Generator("cuda").manual_seed(M)).bfloat16()
    q, s = torch.empty(M, D, dtype=torch.uint8, device="cuda"), torch.empty(M, (D + 31) // 32, dtype=torch.uint8, device="cuda")
    gpu.avits_ckpt8_pack(x, q, s)
    codes, e = oracle.hold(x.double().cpu().numpy(), 8)
    assert np.array_equal(q.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), oracle.ckpt_scales(e))
    out = torch.empty_like(x)
    gpu.avits_ckpt8_unpack(q, s, out)
    assert torch.equal(out.cpu(), torch.from_numpy(oracle.held_values(codes, e, 8)).bfloat16())

"""Logits of up to 2^30 in size, of any mantissa: their product with log2 e is rounded, by up to 64, in the running maximum."""
import pytest

from _sparse import forward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,M,N", [(2, 300, 300), (1, 5, 3000), (1, 1, 1)])
@pytest.mark.parametrize("size", [1.296875, -1.296875, 1.7265625, -1.9921875])
def test_equal_logits(gpu, H, M, N, size, dtype):
    """The mean of the values."""
    s = make(H, H, 64, (0, M), (0, N), dtype, seed=71, extra=0, packed=False)
    s["q"].zero_()
    s["k"].zero_()
    s["q"][:, :, 0], s["k"][:, :, 0] = 2.0 ** 15, size * 2.0 ** 14
    forward(gpu, s, mask=None, scale=1.0)
    v = s["v"].double()
    # All probabilities are alike, to bf16 one rounding; N additions and a division in fp32, then the result's rounding.
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    size_v = v.abs().mean(0)
    tol = ((N + 2) * 2.0 ** -24 + (half if dtype == "bf16" else 0)) * size_v + half * v.mean(0).abs()
    assert ((s["o"].double() - v.mean(0)).abs() <= 1.01 * tol).all()
    assert ((s["lse"].double() / (size * 2.0 ** 29) - 1).abs() < 2.0 ** -21).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
def test_one_above_the_rest(gpu, sign, dtype):
    """One key of every 300 rows has the largest logit by 2^22: its value, exactly."""
    import torch
    s = make(2, 2, 64, (0, 130), (0, 300), dtype, seed=73, extra=0, packed=False)
    s["q"].zero_()
    s["k"].zero_()
    s["q"][:, :, 0], s["k"][:, :, 0] = 2.0 ** 15, sign * 1.296875 * 2.0 ** 14
    s["k"][211, :, 0] = (sign * 1.296875 + 2.0 ** -7) * 2.0 ** 14
    forward(gpu, s, mask=None, scale=1.0)
    assert torch.equal(s["o"], s["v"][211].expand(130, 2, 64))

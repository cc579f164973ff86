"""Pins of oracle/lowbit.py: grids against their bit patterns, roundings
against a search over all codes, gradients against differences."""
import numpy as np
import pytest

import oracle


def _decode(code, ebits, mbits, bias):
    e, m = code >> mbits & (2 ** ebits - 1), code & (2 ** mbits - 1)
    return m * 2.0 ** (1 - bias - mbits) if e == 0 else (1 + m / 2 ** mbits) * 2.0 ** (e - bias)


def test_grids_are_their_bit_patterns():
    assert list(oracle.E2M1) == [_decode(c, 2, 1, 1) for c in range(8)]
    assert list(oracle.E4M3) == [_decode(c, 4, 3, 7) for c in range(127)]


@pytest.mark.parametrize("bits", [4, 8])
def test_rounding_is_to_the_nearest_code_ties_to_even(bits):
    grid = oracle.E2M1 if bits == 4 else oracle.E4M3
    mids = (grid[1:] + grid[:-1]) / 2
    a = np.concatenate([grid, mids, np.nextafter(mids, 0), np.nextafter(mids, 9e9), [grid[-1] * 1.7]])
    got = oracle.nearest_code(a, grid)
    for v, c in zip(a, got):
        d = np.abs(grid - v)
        best = np.flatnonzero(d == d.min())
        assert c in best and (len(best) == 1 or c % 2 == 0), (v, c, best)


def test_scales():
    x = np.zeros((6, 64))
    x[0, 3], x[0, 40] = 6.0, 7.99          # both exponent 2: scale 1
    x[1, 0], x[1, 33] = 448.0, 448.1       # 8 bits: 1, then 2
    x[2, 5] = np.inf
    x[3, 1] = 2.0 ** -130
    x[4, 0], x[4, 32] = 3.999, 4.0
    assert oracle.block_exponents(x, 4).tolist() == [[0, 0], [6, 6], [128, -127], [-127, -127], [-1, 0], [-127, -127]]
    e8 = oracle.block_exponents(x, 8)
    assert e8[1].tolist() == [0, 1] and e8[2, 0] == 128 and e8[5].tolist() == [-127, -127]


def test_held_values_are_within_half_a_step():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((7, 77)) * np.exp2(rng.integers(-20, 20, (7, 77)))
    c, e = oracle.hold(x, 8)
    v = oracle.held_values(c, e, 8)
    s = np.repeat(2.0 ** e, 32, axis=1)[:, :77]
    assert (np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10)).all()
    c, e = oracle.hold(x, 4)
    v = oracle.held_values(c, e, 4)
    s = np.repeat(2.0 ** e, 32, axis=1)[:, :77]
    # Half a step is a quarter of the value at most (2 to 3 and 4 to 6), 0.25 scales below 1;
    # 6 to 8 scales become 6.
    assert (np.abs(v - x) <= np.maximum(np.abs(x) / 4, s / 4)).all()


def test_the_four_bit_layout():
    c = (np.arange(3 * 96).reshape(3, 96) % 16).astype(np.uint8)
    e = np.arange(9).reshape(3, 3)
    q, s = oracle.mx_pack(c, e)
    assert q.shape == (3, 48) and s.shape == (2, 8, 2)
    assert q[1, 5] == c[1, 10] + 16 * c[1, 11]
    assert s[1, 2, 0] == 127 + e[2, 2] and s[0, 1, 1] == 127 + e[1, 1] and s[1, 2, 1] == 0
    c2, e2 = oracle.mx_unpack(q, s)
    assert np.array_equal(c, c2) and np.array_equal(e, e2)


def test_gradients_against_differences():
    rng = np.random.default_rng(6)
    off = [0, 2, 2, 5]
    x, dh = rng.standard_normal((5, 6)) + 0.5, rng.standard_normal((5, 6))
    sh, sc = rng.standard_normal((3, 6)), rng.standard_normal((3, 6))
    loss = lambda x, sh, sc: (oracle.norm_forward(x, sh, sc, off, 1e-6)[0] * dh).sum()  # noqa: E731
    _, mean, rstd = oracle.norm_forward(x, sh, sc, off, 1e-6)
    grads = oracle.norm_backward(dh, x, mean, rstd, sc, off)
    for at, (arg, g) in enumerate(((0, grads[0]), (2, grads[1]), (1, grads[2]))):
        args = [x, sh, sc]
        num = np.zeros_like(args[arg])
        for i in np.ndindex(num.shape):
            up, dn = [a.copy() for a in args], [a.copy() for a in args]
            up[arg][i] += 1e-6
            dn[arg][i] -= 1e-6
            num[i] = (loss(*up) - loss(*dn)) / 2e-6
        # The second difference term is 1e-12 of O(10) derivatives; the cancellation 1e-16 * O(10) / 1e-6.
        assert np.abs(num - g).max() < 1e-7, at
    v = np.linspace(-7, 7, 57)
    num = (oracle.gelu_tanh(v + 1e-6) - oracle.gelu_tanh(v - 1e-6)) / 2e-6
    assert np.abs(num - oracle.gelu_slope(v)).max() < 1e-8

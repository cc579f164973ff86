"""Pins of oracle/attend.py: the rotation against complex products and the block's
own, gradients against differences, the choice against a search, the mask's bits."""
import numpy as np
import pytest

import oracle


def _r(*shape, seed=0):
    return np.random.default_rng(seed).standard_normal(shape)


def test_rotation_is_the_blocks_own():
    pos = np.random.default_rng(1).integers(0, 90, (11, 3))
    x = _r(11, 3, 64)
    dims = (8, 28, 28)
    freq = np.concatenate([10000.0 ** (-2.0 * np.arange(n // 2) / n) for n in dims])
    want = oracle.apply_rope(x, oracle.rope_angles(pos * 0.5, 64))
    assert np.allclose(oracle.turn(x, oracle.rope_turns(pos, freq, dims, 0.5), False), want, atol=1e-12)


@pytest.mark.parametrize("halves", [False, True])
def test_rotation_is_a_complex_product(halves):
    x, a = _r(5, 2, 64), _r(5, 10)
    y = oracle.turn(x, a, halves)
    i, j = oracle.pair_index(20, halves)
    assert np.allclose(y[..., i] + 1j * y[..., j], (x[..., i] + 1j * x[..., j]) * np.exp(1j * a)[:, None])
    assert np.array_equal(y[..., 20:], x[..., 20:])


@pytest.mark.parametrize("eps", [1e-6, 0.3, 0.0])
def test_norm_gradients_against_differences(eps):
    x, g, dy, a = _r(3, 2, 64), _r(64, seed=1), _r(3, 2, 64, seed=2), _r(3, 20, seed=3)
    gg = g if eps else None
    dx, dg = oracle.norm_turn_backward(dy, x, gg, eps, a, True)
    f = lambda x, g: (oracle.norm_turn(x, g, eps, a, True) * dy).sum()  # noqa: E731
    step, way = 1e-6, _r(3, 2, 64, seed=4)
    assert abs((f(x + step * way, gg) - f(x - step * way, gg)) / (2 * step) - (dx * way).sum()) < 1e-7 * np.abs(dx * way).sum()
    if eps:
        way = _r(64, seed=5)
        assert abs((f(x, g + step * way) - f(x, g - step * way)) / (2 * step) - (dg * way).sum()) < 1e-7 * np.abs(dg * way).sum()


def test_choice():
    q_off, k_off = (0, 130, 130, 300), (0, 200, 200, 700)
    qm, km = oracle.block_means(_r(300, 4, 64), q_off, 128), oracle.block_means(_r(700, 2, 64, seed=1), k_off, 64)
    assert qm.shape == (4, 4, 64) and km.shape == (12, 2, 64)
    on = oracle.block_select(qm, km, 2, q_off, k_off, q_lead=1, k_lead=65)
    assert on.shape == (4, 4, 8)
    assert on[:, 0, :4].all() and not on[:, 0, 4:].any() and on[:, 2].all()     # first blocks hold leading rows
    for h in range(4):
        s = km[4:, h // 2] @ qm[3, h]
        rest = sorted(range(2, 8), key=lambda j: -s[j])[:2]
        assert sorted(np.flatnonzero(on[h, 3])) == sorted([0, 1] + rest)
    same = oracle.block_select(np.zeros_like(qm), km, 3, q_off, k_off)
    assert same[:, :2, :3].all() and same[:, 2:, :3].all() and same.sum() == 3 * 16     # ties: the lowest
    bad = km.copy()
    bad[4] = np.nan
    assert not oracle.block_select(qm, bad, 7, q_off, k_off)[:, 2:, 0].any()


def test_words():
    on = np.zeros((2, 1, 70), bool)
    on[0, 0, [0, 63, 69]] = on[1, 0, 64] = True
    w = oracle.words(on, 3)
    assert w.shape == (2, 1, 3) and w[0, 0].tolist() == [1 - (1 << 63), 32, 0] and w[1, 0].tolist() == [0, 1, 0]


def test_attention_is_the_blocks_own_where_all_is_kept():
    q, k, v = _r(140, 2, 64), _r(140, 2, 64, seed=1), _r(140, 2, 64, seed=2)
    o, lse = oracle.sparse_attention(q, k, v, oracle.allowed(None, (0, 140), (0, 140), 140, 140), 64 ** -0.5)
    want, want_lse = oracle.attention(q, k, v)
    assert np.allclose(o, want.reshape(o.shape)) and np.allclose(lse, want_lse)


def test_attention_gradients_against_differences():
    q_off, k_off = (0, 140, 150), (0, 100, 230)
    q, k, v, do = _r(150, 4, 8), _r(230, 2, 8, seed=1), _r(230, 2, 8, seed=2), _r(150, 4, 8, seed=3)
    on = np.random.default_rng(4).random((4, 3, 3)) < 0.6
    on[1, 1] = False
    ok = oracle.allowed(on, q_off, k_off, 150, 230)
    assert not ok[:, :140, 100:].any() and not ok[1, 128:140].any()
    o, lse = oracle.sparse_attention(q, k, v, ok, 0.3)
    assert (o[128:140, 1] == 0).all() and (lse[1, 128:140] == -np.inf).all()
    g = oracle.sparse_attention_backward(do, q, k, v, o, lse, ok, 0.3)
    x = [q, k, v]
    for i in range(3):
        way = _r(*x[i].shape, seed=5 + i)
        up, dn = list(x), list(x)
        up[i], dn[i] = x[i] + 1e-6 * way, x[i] - 1e-6 * way
        num = ((oracle.sparse_attention(*up, ok, 0.3)[0] - oracle.sparse_attention(*dn, ok, 0.3)[0]) * do).sum() / 2e-6
        assert abs(num - (g[i] * way).sum()) < 1e-6 * np.abs(g[i] * way).sum(), i

"""Norm and rotation of queries and keys, and the backward pass, element by element
within bounds from the arithmetic."""
import numpy as np
import pytest

import oracle
from _bounds import assert_within
from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}
# Sine and cosine: fp32 the library's (2 ulp and the fraction's rounding, 2 pi 2^-25);
# bf16 the instruction's, taken to 2^-18 here (a 2^10th of a half step of bf16).
TURN = {"f32": 2.0 ** -22, "bf16": 2.0 ** -18}


def _np(t):
    return t.double().cpu().numpy()


def _make(M, H, Hk, d, dtype, layout, dims, seed=0, eps=1e-6, gains=True, far=60, packed=True, odd=0):
    """Inputs as columns of one buffer (rows at any element with odd > 0)."""
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = TORCH_DT[dtype]

    def columns():
        ld = (H + 2 * Hk) * d + odd
        buf = (torch.randn(max(M, 1) * ld + odd, generator=g)).to(dt).cuda()[odd:odd + M * ld].view(M, ld) if M else \
            torch.empty(0, ld, dtype=dt, device="cuda")
        x = buf[:, :(H + 2 * Hk) * d].unflatten(1, (H + 2 * Hk, d))
        q, k, _ = x.split([H, Hk, Hk], 1)
        return q, k
    s = dict(q=columns() if packed else None, dy=columns(), out=columns(), eps=eps, layout=layout, dims=dims, pos_scale=0.5)
    s["g"] = [(1 + 0.3 * torch.randn(d, generator=g)).to(dt).cuda() if gains else None for _ in range(2)]
    s["pos"] = torch.randint(-far, far, (M, len(dims)), generator=g, dtype=torch.int32).cuda()
    import paper_2608_17995_amd as avits
    s["freq"] = avits.avits_rope_frequencies(dims).cuda()
    return s


def _kw(s):
    return dict(eps=s["eps"], pos=s["pos"], freq=s["freq"], dims=s["dims"], pos_scale=s["pos_scale"], layout=s["layout"],
                g_q=s["g"][0], g_k=s["g"][1])


def _other(v, rot, halves):
    """The magnitude of both elements of each element's pair."""
    a, b = oracle.pair_index(rot, halves)
    out = np.abs(v)
    out[..., a] = out[..., b] = np.abs(v[..., a]) + np.abs(v[..., b])
    return out


def _check_forward(s, dtype, got):
    ang = oracle.rope_turns(s["pos"].cpu().numpy(), s["freq"].cpu().numpy(), s["dims"], s["pos_scale"])
    halves, rot = bool(s["layout"]), sum(s["dims"])
    for x, g, y in zip(s["x"], s["g"], got):
        g = None if g is None else _np(g)
        want = oracle.norm_turn(x, g, s["eps"], ang, halves)
        size = _other(oracle.norm_turn(x, g, s["eps"], None, halves), rot, halves)
        # n: half of 12 roundings of the sum, 2 of the root, 1 of the product; the gain, two products, a sum: 4.
        err = (14 * U + TURN[dtype]) * size
        assert_within(_np(y), want, err + HALF[dtype] * (np.abs(want) + err))


def _check_backward(s, dtype, dx, dg):
    ang = oracle.rope_turns(s["pos"].cpu().numpy(), s["freq"].cpu().numpy(), s["dims"], s["pos_scale"])
    halves, rot = bool(s["layout"]), sum(s["dims"])
    for x, g, dy, got, gg in zip(s["x"], s["g"], s["dyv"], dx, dg):
        gain = None if g is None else _np(g)
        want, wg = oracle.norm_turn_backward(dy, x, gain, s["eps"], ang, halves)
        e = _other(dy, rot, halves)
        if s["eps"] > 0:
            r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + s["eps"])
            n = np.abs(x * r)
            eg = e * (1 if gain is None else np.abs(gain))
            # The turn back 3, n 10, the average 12 more, the products and the difference 6.
            err = (31 * U + TURN[dtype]) * r * (eg + n * (eg * n).mean(-1, keepdims=True))
        else:
            err = (3 * U + TURN[dtype]) * e
        assert_within(_np(got), want, err + HALF[dtype] * (np.abs(want) + err), "dx")
        if gg is not None:
            # A lane's chain of rows (at most rows / 2048 of them, each with its heads), 8 steps between
            # lanes and waves, then 512 / 8 + 8 partial sums; each term off by 14 roundings and the turn.
            chain = 96 + (len(x) // 2048 + 1) * 40
            assert_within(_np(gg), wg, ((chain + 14) * U + TURN[dtype]) * (e * n).sum((0, 1)), "dg")


SHAPES = [(1, 16, 16, 128, (16, 56, 56)), (1, 3, 1, 64, (64,)), (7, 5, 5, 64, (8, 28, 28)), (67, 6, 2, 128, (44,)),
          (33, 1, 1, 64, (6, 0, 22)), (389, 6, 2, 64, (44,)), (130, 9, 3, 128, (128,)), (2, 40, 8, 128, (2,)), (300, 2, 1, 64, (4, 4, 6, 2))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("M,H,Hk,d,dims", SHAPES)
def test_both_ways(gpu, M, H, Hk, d, dims, layout, dtype, odd):
    import torch
    s = _make(M, H, Hk, d, dtype, layout, dims, odd=odd)
    s["x"], s["dyv"] = [_np(t) for t in s["q"]], [_np(t) for t in s["dy"]]
    gpu.avits_qk_norm_rope(*s["q"], *s["out"], **_kw(s))
    _check_forward(s, dtype, s["out"])
    dg = [torch.empty(d, device="cuda") for _ in range(2)]
    gpu.avits_qk_norm_rope_backward(*s["dy"], *s["q"], *s["out"], *dg, **_kw(s))
    _check_backward(s, dtype, s["out"], dg)
    # In place, and over the gradient that came in.
    gpu.avits_qk_norm_rope_backward(*s["dy"], *s["q"], *s["dy"], **_kw(s))
    for a, b in zip(s["dy"], s["out"]):
        assert torch.equal(a, b)
    gpu.avits_qk_norm_rope(*s["q"], *s["q"], **_kw(s))
    _check_forward(s, dtype, s["q"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [0, 1])
def test_many_rows(gpu, layout, dtype):
    """More rows than waves: several to a wave."""
    import torch
    s = _make(5003, 3, 2, 64, dtype, layout, (24, 40))
    s["x"], s["dyv"] = [_np(t) for t in s["q"]], [_np(t) for t in s["dy"]]
    gpu.avits_qk_norm_rope(*s["q"], *s["out"], **_kw(s))
    _check_forward(s, dtype, s["out"])
    dg = [torch.empty(64, device="cuda") for _ in range(2)]
    gpu.avits_qk_norm_rope_backward(*s["dy"], *s["q"], *s["out"], *dg, **_kw(s))
    _check_backward(s, dtype, s["out"], dg)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_alone(gpu, dtype):
    """Queries or keys alone, no norm, no gains, no rotation."""
    import torch
    s = _make(21, 4, 2, 64, dtype, 0, (64,), gains=False)
    s["x"], s["dyv"] = [_np(t) for t in s["q"]], [_np(t) for t in s["dy"]]
    gpu.avits_qk_norm_rope(s["q"][0], None, s["out"][0], None, **_kw(s))
    gpu.avits_qk_norm_rope(None, s["q"][1], None, s["out"][1], **_kw(s))
    _check_forward(s, dtype, s["out"])
    s["eps"] = 0.0
    gpu.avits_qk_norm_rope(*s["q"], *s["out"], **_kw(s))
    _check_forward(s, dtype, s["out"])
    gpu.avits_qk_norm_rope_backward(*s["dy"], None, None, *s["out"], **_kw(s))
    _check_backward(s, dtype, s["out"], (None, None))
    # Neither: a copy, whatever the values.
    x = s["q"][0].clone()
    x[0, 0, 0], x[1, 1, 1] = float("nan"), float("inf")
    o = torch.empty_like(x)
    gpu.avits_qk_norm_rope(x, None, o, None, eps=0.0)
    assert torch.equal(o.view(torch.int16 if dtype == "bf16" else torch.int32), x.view(torch.int16 if dtype == "bf16" else torch.int32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_positions(gpu, dtype):
    """Angles of positions up to 2^31 lose nothing."""
    import torch
    s = _make(64, 2, 1, 128, dtype, 1, (128,))
    s["pos"] = torch.randint(-2 ** 31, 2 ** 31 - 1, (64, 1), generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    s["x"] = [_np(t) for t in s["q"]]
    # In 64 bits an angle of 2^31 is itself off by 2^31 2^-53 of itself in oracle and kernel alike: 2^-20.
    turn, TURN[dtype] = TURN[dtype], TURN[dtype] + 2.0 ** -20
    try:
        gpu.avits_qk_norm_rope(*s["q"], *s["out"], **_kw(s))
        _check_forward(s, dtype, s["out"])
    finally:
        TURN[dtype] = turn


def test_gradient_against_differences(gpu):
    import torch
    s = _make(40, 3, 1, 64, "f32", 1, (40,))
    dg = [torch.empty(64, device="cuda") for _ in range(2)]
    gpu.avits_qk_norm_rope_backward(*s["dy"], *s["q"], *s["out"], *dg, **_kw(s))
    dx = [t.clone() for t in s["out"]]

    def loss(q, g):
        out = [torch.empty_like(t) for t in q]
        gpu.avits_qk_norm_rope(*q, *out, **{**_kw(s), "g_q": g[0], "g_k": g[1]})
        return sum((o.double() * d.double()).sum() for o, d in zip(out, s["dy"]))
    for i in range(2):
        for leaf, grad in ((s["q"], dx), (s["g"], dg)):
            step = 0.01 * leaf[i].double().norm() / grad[i].double().norm()
            up, dn = list(leaf), list(leaf)
            up[i], dn[i] = (leaf[i] + step * grad[i]).float(), (leaf[i] - step * grad[i]).float()
            f = (lambda t: loss(t, s["g"])) if leaf is s["q"] else (lambda t: loss(s["q"], t))
            # The third derivative's share of a step of one percent is 1e-4; fp32 sums 1e-5.
            assert abs((f(up) - f(dn)) / (2 * step) / grad[i].double().square().sum() - 1) < 1e-3


def test_bad_values_stay_in_their_head(gpu):
    import torch
    s = _make(9, 4, 2, 64, "bf16", 0, (64,))
    gpu.avits_qk_norm_rope(*s["q"], *s["out"], **_kw(s))
    clean = [t.clone() for t in s["out"]]
    s["q"][0][3, 1, 5], s["q"][1][4, 0, 0] = float("inf"), float("nan")
    gpu.avits_qk_norm_rope(*s["q"], *s["out"], **_kw(s))
    for t, c, (r, h) in zip(s["out"], clean, ((3, 1), (4, 0))):
        same = (t == c).all(-1)
        assert not same[r, h] and same.sum() == same.numel() - 1 and torch.isnan(t[r, h]).any()


def test_no_rows(gpu):
    import torch
    s = _make(0, 4, 2, 64, "bf16", 0, (64,))
    gpu.avits_qk_norm_rope(*s["q"], *s["out"], **_kw(s))
    dg = [torch.ones(64, device="cuda") for _ in range(2)]
    gpu.avits_qk_norm_rope_backward(*s["dy"], *s["q"], *s["out"], *dg, **_kw(s))
    assert not dg[0].any() and not dg[1].any()


def test_same_result_each_time_and_in_a_graph(gpu):
    import torch
    s = _make(3001, 8, 2, 128, "bf16", 0, (16, 56, 56))
    ws = torch.empty(gpu.avits_qk_norm_rope_backward_workspace_bytes(3001, 8, 2, 128), dtype=torch.uint8, device="cuda")
    dg = [torch.empty(128, device="cuda") for _ in range(2)]

    def both():
        gpu.avits_qk_norm_rope_backward(*s["dy"], *s["q"], *s["out"], *dg, workspace=ws, **_kw(s))
    both()
    want = [t.clone() for t in (*s["out"], *dg)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in (*s["out"], *dg):
            t.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((*s["out"], *dg), want):
            assert torch.equal(a, b)

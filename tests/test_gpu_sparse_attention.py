"""Attention over chosen key blocks, and its backward pass, element by element within
bounds from the arithmetic."""
import numpy as np
import pytest

import oracle
from _sparse import backward, check_backward, check_forward, forward, make, np64

pytestmark = pytest.mark.gpu

# H, Hk, d, q_off, k_off
SHAPES = [
    (1, 1, 64, (0, 1), (0, 1)), (2, 1, 128, (0, 1), (0, 333)), (4, 4, 64, (0, 288), (0, 288)), (6, 2, 64, (0, 333), (0, 333)),
    (3, 3, 128, (0, 129), (0, 129)), (2, 2, 128, (0, 700), (0, 700)), (2, 1, 64, (0, 127), (0, 65)), (4, 2, 128, (0, 3), (0, 900)),
    (2, 2, 64, (0, 200, 200, 333), (0, 200, 200, 333)), (4, 1, 128, (0, 130, 190), (0, 70, 400)), (2, 2, 64, (0, 60, 200), (0, 0, 90)),
    (2, 2, 64, (0, 0, 70), (0, 100, 190)), (1, 1, 128, tuple(range(0, 321, 20)), tuple(range(0, 801, 50))), (8, 1, 64, (0, 260), (0, 260)),
    (1, 1, 64, (0, 140), (0, 4300)), (1, 1, 128, (0, 5), (0, 9000)),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d,q_off,k_off", SHAPES)
def test_both_ways(gpu, H, Hk, d, q_off, k_off, dtype):
    s = make(H, Hk, d, q_off, k_off, dtype)
    forward(gpu, s)
    check_forward(s)
    backward(gpu, s)
    check_backward(s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("density", [0.0, 0.03, 1.0, None])
@pytest.mark.parametrize("d", [64, 128])
def test_densities(gpu, d, density, dtype):
    """No block at all, single ones, every one, and no mask."""
    s = make(3, 1, d, (0, 300, 500), (0, 300, 500), dtype, seed=5, density=density or 0.0)
    kw, on = {}, "mask"
    if density == 1.0:
        s["on"][:] = True
        s["mask"][:] = -1
    if density is None:
        kw, on = dict(mask=None), None
    forward(gpu, s, **kw)
    check_forward(s, on)
    backward(gpu, s, **kw)
    check_backward(s, on)
    if density == 0.0:
        assert not s["dq"][:500].any() and not s["dk"][:500].any() and not s["dv"][:500].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_logits(gpu, dtype):
    """Logits in the hundreds, rising and falling along the keys: the running maximum moves."""
    import torch
    s = make(2, 2, 64, (0, 200), (0, 640), dtype, seed=7, density=0.8)
    ramp = torch.linspace(-1, 1, 643, device="cuda")[:, None, None]
    s["k"].copy_((s["k"].float() * 2 + 4 * torch.cat([ramp[:, :, :], -ramp], 1) * s["q"][:1].float().mean()).to(s["k"].dtype))
    s["q"].mul_(8)
    forward(gpu, s)
    check_forward(s)
    backward(gpu, s)
    check_backward(s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_masked_is_not_read(gpu, dtype):
    """NaN and infinities in keys and values that no block keeps, behind a sequence's
    last key, and in rows behind the last sequence, change nothing."""
    s = make(2, 2, 128, (0, 130, 250), (0, 200, 390), dtype, seed=9)
    s["on"][:, :, 1] = False
    s["mask"].copy_(__import__("torch").from_numpy(oracle.words(s["on"], s["mask"].shape[2]).copy()))
    forward(gpu, s)
    backward(gpu, s)
    keep = [np64(s[n]).copy() for n in ("o", "dq", "dk", "dv")]
    for t in (s["k"], s["v"]):
        for rows in (slice(64, 128), slice(264, 328), slice(390, None)):
            t[rows] = float("nan")
        t[64] = float("inf")
    for t in (s["q"], s["do"]):
        t[250:] = float("nan")
    forward(gpu, s)
    backward(gpu, s)
    for n, was in zip(("o", "dq", "dk", "dv"), keep):
        assert np.array_equal(np64(s[n]), was), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_neighbours_bad_keys_stay_theirs(gpu, dtype):
    """A NaN key of one sequence reaches that sequence's rows only, though its tile's rows
    are neighbours in memory."""
    import torch
    s = make(1, 1, 64, (0, 100, 230), (0, 90, 200), dtype, seed=11, density=1.0)
    s["on"][:] = True
    s["mask"][:] = -1
    s["k"][90:200] = float("nan")
    s["v"][90:200] = float("inf")
    forward(gpu, s)
    assert torch.isfinite(s["o"][:100]).all() and torch.isnan(s["o"][100:230]).all()
    s["q"][100:230] = float("nan")
    backward(gpu, s)
    assert torch.isfinite(s["dq"][:100]).all() and torch.isfinite(s["dk"][:90]).all() and torch.isfinite(s["dv"][:90]).all()


def test_gradient_against_differences(gpu):
    import torch
    s = make(4, 2, 64, (0, 150, 290), (0, 150, 290), "f32", seed=13)
    forward(gpu, s)
    backward(gpu, s)
    grads = {n: s["d" + n][:290].double() for n in "qkv"}

    def loss():
        forward(gpu, s)
        return (s["o"][:290].double() * s["do"][:290].double()).sum()
    for n in "qkv":
        leaf = s[n].clone()
        step = 0.01 * leaf[:290].double().norm() / grads[n].norm()
        f = []
        for sign in (1, -1):
            s[n][:290] = (leaf[:290].double() + sign * step * grads[n]).float()
            f.append(loss())
        s[n].copy_(leaf)
        # A step of one percent leaves 1e-4 of the third derivative; fp32 sums 1e-5.
        assert abs((f[0] - f[1]) / (2 * step) / grads[n].square().sum() - 1) < 2e-3, n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_result_each_time_and_in_a_graph(gpu, dtype):
    """Twice the same bits; two graphs that share a workspace, replayed in turn."""
    import torch
    parts = [make(4, 2, 128, (0, 700), (0, 700), dtype, seed=s) for s in (15, 16)]
    code = gpu.BF16 if dtype == "bf16" else gpu.F32
    n = max(gpu.avits_sparse_attention_workspace_bytes(703, 703, 1, 4, 128, code),
            gpu.avits_sparse_attention_backward_workspace_bytes(703, 703, 1, 4, 2, 128, code))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    want, graphs = [], []
    for s in parts:
        forward(gpu, s, workspace=ws)
        backward(gpu, s, workspace=ws)
        want.append([s[n].clone() for n in ("o", "lse", "dq", "dk", "dv")])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            forward(gpu, s, workspace=ws)
            backward(gpu, s, workspace=ws)
        graphs.append(g)
    for _ in range(3):
        for s in parts:
            for n in ("o", "lse", "dq", "dk", "dv"):
                s[n].fill_(5)      # rows behind the last sequence hold it already
        ws.fill_(255)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, w in zip(parts, want):
            for n, t in zip(("o", "lse", "dq", "dk", "dv"), w):
                assert torch.equal(s[n], t), n


def test_other_stream(gpu):
    import torch
    s = make(2, 2, 64, (0, 500), (0, 500), "bf16", seed=17)
    forward(gpu, s)
    backward(gpu, s)
    want = [s[n].clone() for n in ("o", "dq", "dk", "dv")]
    side = torch.cuda.Stream()
    for t in (s[n] for n in ("o", "dq", "dk", "dv")):
        t.fill_(1)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        forward(gpu, s)
    backward(gpu, s, stream=side)
    side.synchronize()
    for n, t in zip(("o", "dq", "dk", "dv"), want):
        assert torch.equal(s[n][:500], t[:500]), n


def test_against_the_dense_statistics(gpu):
    """With every block kept, the log-sum-exp of avits_joint_lse."""
    import torch
    s = make(4, 4, 128, (0, 300), (0, 300), "bf16", seed=19, extra=0, packed=False)
    s["k"] = s["k"].contiguous()
    forward(gpu, s, mask=None)
    lse = torch.empty(4, 300, device="cuda")
    gpu.avits_joint_lse(s["q"].contiguous(), s["k"], lse)
    # Each is within d + 50 roundings of logits of about 4.
    assert (lse - s["lse"]).abs().max() < 200 * 4 * 2.0 ** -24


def test_no_rows(gpu):
    import torch
    for q_off, k_off in (((0, 0), (0, 5)), ((0, 5), (0, 0)), ((0, 0), (0, 0))):
        s = make(2, 1, 64, q_off, k_off, "bf16", extra=0)
        forward(gpu, s)
        backward(gpu, s)
        assert not s["o"].any() and not s["dq"].any() and not s["dk"].any() and not s["dv"].any() and (s["lse"] == -np.inf).all()

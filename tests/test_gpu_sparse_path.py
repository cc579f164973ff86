"""SparseAttention: norm and rotation, choice of key blocks and attention together, and their gradients."""
import numpy as np
import pytest

import oracle
from _bounds import assert_within
from _gpu import TORCH_DT
from _sparse import check_backward, check_forward, np64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}


def _path(H, Hk, d, rows, dtype, seed=0, wide=0, **kw):
    """The object, a projection's output (columns of wider rows with wide > 0), positions, out, dout, dqkv."""
    import torch
    from paper_2608_17995_amd.step import SparseAttention
    g = torch.Generator().manual_seed(seed)
    dt = TORCH_DT[dtype]
    gains = [(1 + 0.3 * torch.randn(d, generator=g)).to(dt).cuda() for _ in range(2)]
    kw = {**dict(dims=(8, 28, 28) if d == 64 else (16, 56, 56), keep=2, tune=True), **kw}
    path = SparseAttention(rows, H, d, Hk=Hk, g_q=gains[0], g_k=gains[1], dtype=dt, **kw)
    cols = (H + 2 * Hk) * d
    qkv = torch.randn(rows, cols + wide, generator=g).to(dt).cuda()[:, :cols]
    pos = torch.randint(0, 40, (rows, 3), generator=g, dtype=torch.int32).cuda()
    dout = torch.randn(rows, H, d, generator=g).to(dt).cuda()
    out = torch.full((rows, H, d), 5.0, dtype=dt, device="cuda")
    return path, qkv, pos, dout, out, torch.full_like(qkv, 5.0)


def _stages(path, qkv, off):
    """The buffers as the helpers of the operators' tests take them."""
    H, Hk, d, M = path.H, path.Hk, path.d, len(qkv)
    q, k, v = qkv.view(M, -1, d).split([H, Hk, Hk], 1)
    return q, k, dict(q=path._q[:M], k=path._k[:M], v=v, q_off=off, k_off=off, scale=d ** -0.5, lse=path._row_lse)


SHAPES = [(4, 4, 128, (0, 700), 64), (6, 2, 64, (0, 1, 1, 400, 900), 100), (2, 1, 128, (0, 77), 0), (16, 16, 64, (0, 1500), 200),
          (1, 1, 64, (0, 1), 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d,off,lead", SHAPES)
def test_stages(gpu, H, Hk, d, off, lead, dtype):
    """Each stage from what the one before left, the gradients through all of them, rows behind the last sequence untouched."""
    import torch
    rows = off[-1] + 3
    path, qkv, pos, dout, out, dqkv = _path(H, Hk, d, rows, dtype, seed=3, wide=64, batch=len(off) - 1, lead=lead)
    path._q.fill_(5)
    path._k.fill_(5)
    path._lse.fill_(5)
    path.forward(qkv, pos, out, off=off, pos_scale=0.5)
    m = off[-1]
    q, k, s = _stages(path, qkv, off)
    ang = oracle.rope_turns(pos.cpu().numpy()[:m], path._freq.cpu().numpy(), path.dims, 0.5)
    for x, g, y in ((q, path.g_q, s["q"]), (k, path.g_k, s["k"])):
        want = oracle.norm_turn(np64(x[:m]), np64(g), 1e-6, ang, False)
        size = np.abs(oracle.norm_turn(np64(x[:m]), np64(g), 1e-6, None, False))
        n = 2 * (sum(path.dims) // 2)
        size[..., :n] = np.repeat(size[..., 0:n:2] + size[..., 1:n:2], 2, -1)
        # 14 roundings in fp32; sine and cosine to 2^-22, in bf16 2^-18.
        err = (14 * U + (2.0 ** -22 if dtype == "f32" else 2.0 ** -18)) * size
        assert_within(np64(y[:m]), want, err + HALF[dtype] * (np.abs(want) + err), "norm and rotation")
        assert (y[m:] == 5).all()
    means = [oracle.block_means(np64(s[n]), off, b) for n, b in (("q", 128), ("k", 64))]
    for ref, got in zip(means, (path._qm, path._km)):
        # 127 additions and a division in 64 bits of magnitudes below 16.
        assert_within(np64(got[:len(ref)]), ref, 130 * 16 * 2.0 ** -53, "means")
    on = oracle.block_select(np64(path._qm[:len(means[0])]), np64(path._km[:len(means[1])]), 2, off, off, lead, lead)
    assert np.array_equal(path._kept.cpu().numpy(), oracle.words(on, path._kept.shape[-1]))
    check_forward(dict(s, o=out, on=on, dtype=dtype))

    # The attention's gradients, then the norm's from the values that they had in the path.
    part = dict(s, o=out, on=on, dtype=dtype, do=dout, dq=torch.full_like(s["q"], 5), dk=torch.full_like(s["k"], 5),
                dv=torch.full_like(s["k"], 5))
    gpu.avits_sparse_attention_backward(dout, s["q"], s["k"], s["v"], out, s["lse"], part["dq"], part["dk"], part["dv"], path._kept,
                                        q_off=off, k_off=off)
    check_backward(part)
    dg = [torch.full((d,), 5.0, device="cuda") for _ in range(2)]
    path.backward(dout, qkv, pos, out, dqkv, *dg)
    dq, dk, dv = dqkv.view(rows, -1, d).split([H, Hk, Hk], 1)
    assert torch.equal(dv, part["dv"]) and (dqkv[m:] == 5).all()
    for got, gg, x, g, dy in ((dq, dg[0], q, path.g_q, part["dq"]), (dk, dg[1], k, path.g_k, part["dk"])):
        x, dy, gain = np64(x[:m]), np64(dy[:m]), np64(g)
        want, wg = oracle.norm_turn_backward(dy, x, gain, 1e-6, ang, False)
        e = np.abs(dy)
        e[..., :n] = np.repeat(e[..., 0:n:2] + e[..., 1:n:2], 2, -1)
        r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6)
        eg, nn = e * np.abs(gain), np.abs(x * r)
        # As in the operator's own test: 31 roundings and the turn; a gain's sum 150 more.
        turn = 2.0 ** -22 if dtype == "f32" else 2.0 ** -18
        err = (31 * U + turn) * r * (eg + nn * (eg * nn).mean(-1, keepdims=True))
        assert_within(np64(got[:m]), want, err + HALF[dtype] * (np.abs(want) + err), "gradient of the projection")
        assert_within(np64(gg), wg, (150 * U + turn) * (e * nn).sum((0, 1)), "gradient of the gain")


def test_gradient_against_differences(gpu):
    """Along its own gradient, with the choice that the forward made."""
    import torch
    path, qkv, pos, dout, out, dqkv = _path(4, 2, 64, 450, "f32", seed=5, lead=40, keep=1)
    dg = [torch.empty(64, device="cuda") for _ in range(2)]
    path.forward(qkv, pos, out)
    path.backward(dout, qkv, pos, out, dqkv, *dg)
    mask = path._kept.clone()

    def loss():
        path.forward(qkv, pos, out)
        assert torch.equal(path._kept, mask), "another choice: the difference says nothing"
        return (out.double() * dout.double()).sum()
    for leaf, grad in ((qkv, dqkv), (path.g_q, dg[0]), (path.g_k, dg[1])):
        old, grad = leaf.clone(), grad.double()
        step = 1e-3 * old.double().norm() / grad.norm()
        f = []
        for sign in (1, -1):
            leaf.copy_((old.double() + sign * step * grad).float())
            f.append(loss())
        leaf.copy_(old)
        # Leaves 1e-6 of the third derivative; the difference of two fp32 losses, 2e-3 of the sum of magnitudes each off by
        # at most 2^-22, 1e-3.
        assert abs((f[0] - f[1]) / (2 * step) / grad.square().sum() - 1) < 2e-3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_graph_other_stream_and_shorter_calls(gpu, dtype):
    """Captured, replayed with eager work between; on another stream; fewer rows than built for."""
    import torch
    path, qkv, pos, dout, out, dqkv = _path(4, 2, 64, 900, dtype, seed=7, lead=64, batch=2)
    dg = [torch.empty(64, device="cuda") for _ in range(2)]
    off = (0, 333, 850)

    def tune(stream=None, off=off, n=900):
        path.forward(qkv[:n], pos[:n], out[:n], off=off, stream=stream)
        path.backward(dout[:n], qkv[:n], pos[:n], out[:n], dqkv[:n], *dg, stream=stream)
    results = (out, dqkv, *dg)

    def clear():
        for t in results:
            t.fill_(5)
    clear()
    tune()
    want = [t.clone() for t in results]
    graph = torch.cuda.CUDAGraph()
    clear()
    with torch.cuda.graph(graph):
        tune()
    for n in (900, 1, 470):
        clear()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want))
        tune(off=None, n=n)                                  # eager work with the same buffers
        first = out[:n].clone()
        path.run(qkv[:n], pos[:n], out[:n])
        assert torch.equal(first, out[:n]) and torch.isfinite(out[:n]).all()
    side = torch.cuda.Stream()
    clear()
    side.wait_stream(torch.cuda.current_stream())
    tune(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(results, want))


def test_no_rotation_and_no_rows(gpu):
    import torch
    path, qkv, _, dout, out, dqkv = _path(2, 2, 64, 200, "bf16", seed=9, dims=None)
    path.forward(qkv, None, out)
    path.backward(dout, qkv, None, out, dqkv)
    want = oracle.norm_turn(np64(qkv.view(200, 6, 64)[:, :2]), np64(path.g_q), 1e-6, None, False)
    assert_within(np64(path._q[:200]), want, (2.0 ** -8 + 2.0 ** -18) * np.abs(want))
    assert torch.isfinite(dqkv).all()
    dg = torch.full((64,), 5.0, device="cuda")
    path.forward(qkv[:0], None, out[:0])
    path.backward(dout[:0], qkv[:0], None, out[:0], dqkv[:0], dg)
    assert (dg == 0).all()


def test_refusals(gpu):
    import torch
    from paper_2608_17995_amd.step import SparseAttention
    for kw in (dict(d=96), dict(H=3, Hk=2), dict(rows=0), dict(batch=0)):
        with pytest.raises(ValueError):
            SparseAttention(**{**dict(rows=128, H=2, d=64, keep=1, dims=(64,)), **kw})
    path, qkv, pos, dout, out, dqkv = _path(2, 2, 64, 130, "bf16", batch=2)
    with pytest.raises(ValueError, match="without a forward"):
        path.backward(dout, qkv, pos, out, dqkv)
    for bad in (dict(off=(0, 5, 9, 12)), dict(off=(0, 140)), dict(off=(0, 9, 5)), dict(off=(1, 9)), dict(off=(0,))):
        with pytest.raises(ValueError):
            path.run(qkv, pos, out, **bad)
    with pytest.raises(ValueError):
        path.run(torch.cat([qkv, qkv]), pos, out)
    with pytest.raises(ValueError):
        path.run(qkv[:, :-64], pos, out)
    path.forward(qkv, pos, out)
    with pytest.raises(ValueError, match="rows"):
        path.backward(dout, qkv[:5], pos, out, dqkv[:5])
    with pytest.raises(ValueError):
        path.forward(qkv, pos, out, off=(0, 140))
    with pytest.raises(ValueError, match="without a forward"):      # a refused forward leaves none
        path.backward(dout, qkv, pos, out, dqkv)
    plain = SparseAttention(130, 2, 64, 1, dims=(8, 28, 28))
    with pytest.raises(ValueError, match="tune"):
        plain.forward(qkv, pos, out)

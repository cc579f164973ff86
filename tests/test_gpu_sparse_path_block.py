"""SparseAttention, every key block kept, between a block's own projections: the block's output, of both kinds of block; and its
gradients with gains for the text rows."""
import numpy as np
import pytest

import oracle
from _gpu import assert_close, dev, double_weights_dev, host
from oracle.block import _modulate, rope_axes
from synth import configs as C
from synth import generator as G
from test_gpu_stages import _block_inputs

pytestmark = pytest.mark.gpu

TINY = [C.TINY_F32, C.TINY_BF16, C.TINY_BF16_REF, C.TINY_F32_RAGGED]
IDS = [w.name for w in TINY]
ALL = 1 << 30     # blocks to keep


def _attend(w, S, p, pos, lead, gains, **kw):
    """The path's output [S, D] for a projection p [S, 3 D], rounded to the workload's type."""
    import torch
    from paper_2608_17995_amd.step import SparseAttention
    from _gpu import TORCH_DT
    d = w.D // w.H
    g = {n: dev(v, w.dtype) for n, v in gains.items()}
    path = SparseAttention(S, w.H, d, ALL, dims=rope_axes(d), lead=lead, dtype=TORCH_DT[w.dtype], **g, **kw)
    out = torch.empty(S, w.H, d, dtype=path.dtype, device="cuda")
    path.run(dev(p, w.dtype), dev(pos), out)
    return path, host(out).reshape(S, -1)


@pytest.mark.parametrize("w", TINY, ids=IDS)
def test_single_block(gpu, w):
    import torch
    x, pos = _block_inputs(w, w.L, w.k, seed=11)
    S, D = x.shape
    ws = G.single_block_weights(w, 0)
    mod, W, b = (np.asarray(ws[n], np.float64) for n in ("mod", "w_in", "b_in"))
    h = _modulate(x, mod[0], mod[1])
    path, o = _attend(w, S, h @ W[:3 * D].T + b[:3 * D], pos, w.L, dict(g_q=ws["g_q"], g_k=ws["g_k"]))
    bw = gpu.BlockWeights(gpu.BLOCK_SINGLE, single=double_weights_dev(ws, w.dtype))
    t_x = dev(x, w.dtype)
    q, k, out = (torch.empty_like(t_x) for _ in range(3))
    gpu.avits_block_qk(t_x, dev(pos), w.L, S - w.L, bw, w.H, q, k)
    assert_close(host(path._q[:S]).reshape(S, -1), host(q), w.dtype, "queries")
    assert_close(host(path._k[:S]).reshape(S, -1), host(k), w.dtype, "keys")
    # The rest of the block in 64 bits around the path's output, against the block's own.
    gpu.avits_block_forward(t_x, out, dev(pos), w.L, S - w.L, bw, w.H)
    y = np.concatenate([o, oracle.gelu_tanh(h @ W[3 * D:].T + b[3 * D:])], 1) @ np.asarray(ws["w_out"], np.float64).T + ws["b_out"]
    assert_close(mod[2] * y, host(out) - x, w.dtype, "block update", fp32_atol=2e-4)     # two sides, each within 1e-4
    assert_close(mod[2] * y, oracle.single_block(x, pos, ws, w.H)[0] - x, w.dtype, "block update")


@pytest.mark.parametrize("w", TINY, ids=IDS)
@pytest.mark.parametrize("n_txt", [None, 0, 1, "all"])
def test_double_block(gpu, w, n_txt):
    import torch
    S = w.L + w.R + w.k
    n_txt = {None: w.L, "all": S}.get(n_txt, n_txt)
    x, pos = _block_inputs(w, n_txt, S - n_txt, seed=13)
    D = w.D
    wt, wi = G.double_stream_weights(w, 0, 0), G.double_stream_weights(w, 0, 1)
    f64 = lambda v: np.asarray(v, np.float64)  # noqa: E731
    parts = [(slice(0, n_txt), wt), (slice(n_txt, S), wi)]
    p = np.concatenate([_modulate(x[r], f64(s["mod"])[0], f64(s["mod"])[1]) @ f64(s["w_qkv"]).T + f64(s["b_qkv"]) for r, s in parts])
    path, o = _attend(w, S, p, pos, n_txt, dict(g_q=wi["g_q"], g_k=wi["g_k"], g_q_text=wt["g_q"], g_k_text=wt["g_k"]))
    bw = gpu.BlockWeights(gpu.BLOCK_DOUBLE, txt=double_weights_dev(wt, w.dtype), img=double_weights_dev(wi, w.dtype))
    t_x = dev(x, w.dtype)
    q, k, out = (torch.empty_like(t_x) for _ in range(3))
    gpu.avits_block_qk(t_x, dev(pos), n_txt, S - n_txt, bw, w.H, q, k)
    assert_close(host(path._q[:S]).reshape(S, -1), host(q), w.dtype, "queries")
    assert_close(host(path._k[:S]).reshape(S, -1), host(k), w.dtype, "keys")
    gpu.avits_block_forward(t_x, out, dev(pos), n_txt, S - n_txt, bw, w.H)
    got = np.empty((S, D))
    for r, s in parts:
        mod = f64(s["mod"])
        y = x[r] + mod[2] * (o[r] @ f64(s["w_o"]).T + f64(s["b_o"]))
        m = oracle.gelu_tanh(_modulate(y, mod[3], mod[4]) @ f64(s["w_mlp1"]).T + f64(s["b_mlp1"]))
        got[r] = y + mod[5] * (m @ f64(s["w_mlp2"]).T + f64(s["b_mlp2"]))
    assert_close(got - x, host(out) - x, w.dtype, "block update", fp32_atol=2e-4)
    assert_close(got - x, oracle.double_block(x, pos, n_txt, wt, wi, w.H)[0] - x, w.dtype, "block update")


def _tuned(dtype, M, lead, seed):
    import torch
    from _gpu import TORCH_DT
    from paper_2608_17995_amd.step import SparseAttention
    g = torch.Generator().manual_seed(seed)
    dt, H, Hk, d = TORCH_DT[dtype], 4, 2, 64
    gains = [(1 + 0.3 * torch.randn(d, generator=g)).to(dt).cuda() for _ in range(4)]
    path = SparseAttention(M + 5, H, d, 1, dims=(8, 28, 28), Hk=Hk, lead=lead, g_q=gains[0], g_k=gains[1], g_q_text=gains[2], g_k_text=gains[3],
                           tune=True, dtype=dt)
    qkv = torch.randn(M, (H + 2 * Hk) * d, generator=g).to(dt).cuda()
    pos = torch.randint(0, 40, (M, 3), generator=g, dtype=torch.int32).cuda()
    dout = torch.randn(M, H, d, generator=g).to(dt).cuda()
    return path, gains, qkv, pos, dout, torch.empty_like(dout), torch.empty_like(qkv), [torch.full((d,), 5.0, device="cuda") for _ in range(4)]


def test_text_gains_against_differences(gpu):
    """Along its own gradient, with the choice that the forward made, in fp32."""
    import torch
    path, gains, qkv, pos, dout, out, dqkv, dg = _tuned("f32", 450, 40, 5)

    def loss():
        path.forward(qkv, pos, out)
        assert torch.equal(path._kept, mask), "another choice: the difference says nothing"
        return (out.double() * dout.double()).sum()
    path.forward(qkv, pos, out)
    mask = path._kept.clone()
    path.backward(dout, qkv, pos, out, dqkv, dg[0], dg[1], dg_q_text=dg[2], dg_k_text=dg[3])
    for leaf, grad in ((qkv, dqkv), *zip(gains, dg)):
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
@pytest.mark.parametrize("M,lead", [(450, 40), (130, 0), (77, 77), (50, 90), (1, 1), (0, 9)])
def test_text_gains_rows(gpu, M, lead, dtype):
    """Each row's gradient is as with its gains for all rows; the two sums of a gain are those of its rows; in a graph too."""
    import torch
    path, gains, qkv, pos, dout, out, dqkv, dg = _tuned(dtype, M, lead, 7)

    def tune():
        path.forward(qkv, pos, out)
        path.backward(dout, qkv, pos, out, dqkv, dg[0], dg[1], dg_q_text=dg[2], dg_k_text=dg[3])
    tune()
    d, text = 64, min(lead, M)
    part = torch.empty_like(qkv)
    dq, dk, dv = part.unflatten(1, (-1, d)).split([4, 2, 2], 1)
    q, k, v = qkv.unflatten(1, (-1, d)).split([4, 2, 2], 1)
    kw = dict(pos=pos, freq=path._freq, dims=path.dims)
    for r, g, s in ((slice(0, text), gains[2:], dg[2:]), (slice(text, M), gains[:2], dg[:2])):
        want = [torch.empty_like(t) for t in (q, k)]
        gpu.avits_qk_norm_rope(q, k, *want, g_q=g[0], g_k=g[1], **kw)
        assert torch.equal(path._q[:M][r], want[0][r]) and torch.equal(path._k[:M][r], want[1][r])
        if M:
            gpu.avits_sparse_attention_backward(dout, path._q[:M], path._k[:M], v, out, path._row_lse, dq, dk, dv, path._kept)
        sums = [torch.empty(d, device="cuda") for _ in range(2)]
        gpu.avits_qk_norm_rope_backward(dq[r], dk[r], q[r], k[r], dq[r], dk[r], *sums, g_q=g[0], g_k=g[1], **{**kw, "pos": pos[r]})
        assert torch.equal(dqkv[r], part[r]) and all(torch.equal(a, b) for a, b in zip(s, sums))
    first = [t.clone() for t in (out, dqkv, *dg)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tune()
    for _ in range(2):
        for t in (out, dqkv, *dg):
            t.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, dqkv, *dg), first))


def test_text_gains_refusals(gpu):
    import torch
    from paper_2608_17995_amd.step import SparseAttention
    one = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="batch = 1"):
        SparseAttention(128, 2, 64, 1, dims=(64,), batch=2, g_k_text=one)
    path = SparseAttention(128, 2, 64, 1, dims=None, tune=True)
    x, o = torch.zeros(9, 6 * 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(9, 2, 64, dtype=torch.bfloat16, device="cuda")
    path.forward(x, None, o)
    with pytest.raises(ValueError, match="text"):
        path.backward(o, x, None, o, x.clone(), dg_q_text=torch.empty(64, device="cuda"))

"""The low-bit and training calls past 32-bit offsets, on streams that are not
the current one without a workspace of the caller's, and captured into graphs
that share one."""
import numpy as np
import pytest

import oracle
from _bounds import assert_within

pytestmark = pytest.mark.gpu


def _np(t):
    return t.double().cpu().numpy()


def _randn(*shape):
    import torch
    return torch.randn(*shape, dtype=torch.bfloat16, device="cuda", generator=torch.Generator("cuda").manual_seed(sum(shape)))


def _held(rng, M, K):
    import torch
    codes, e = oracle.hold(rng.standard_normal((M, K)), 4)
    q, s = oracle.mx_pack(codes, e)
    return torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), oracle.held_values(codes, e, 4)


def test_rows_past_two_to_the_31_elements(gpu):
    """Rows do not depend on each other: the last ones come out as in a call of their own."""
    import torch
    D, M = 2048, (1 << 20) + 37
    x, own = _randn(M, D), slice(M - 37, M)
    xo = x[own].contiguous()
    mod = _randn(2, D)
    h, ho = torch.empty_like(x), torch.empty_like(xo)
    mean, rstd = (torch.empty(M, device="cuda") for _ in range(2))
    gpu.avits_layer_norm(x, mod[0], mod[1], h, mean, rstd)
    gpu.avits_layer_norm(xo, mod[0], mod[1], ho)
    assert torch.equal(h[own], ho)
    q, s = torch.empty(M, D, dtype=torch.uint8, device="cuda"), torch.empty(M, D // 32, dtype=torch.uint8, device="cuda")
    gpu.avits_ckpt8_pack(x, q, s)
    qo, so = torch.empty_like(q[own]), torch.empty_like(s[own])
    gpu.avits_ckpt8_pack(xo, qo, so)
    assert torch.equal(q[own], qo) and torch.equal(s[own], so)
    dx, dxo = torch.empty_like(x), torch.empty_like(xo)
    for held in (dict(x=x), dict(x_q8=q, x_s8=s)):
        gpu.avits_layer_norm_backward(h, mean, rstd, mod[1], dx, dres=x, **held)
        gpu.avits_layer_norm_backward(ho, mean[own].contiguous(), rstd[own].contiguous(), mod[1], dxo, dres=xo,
                                      **{k: v[own].contiguous() for k, v in held.items()})
        assert torch.equal(dx[own], dxo)
    gpu.avits_gelu_backward(h, dx, m_q8=q, m_s8=s)
    gpu.avits_gelu_backward(ho, dxo, m_q8=qo, m_s8=so)
    assert torch.equal(dx[own], dxo)
    gpu.avits_ckpt8_unpack(q, s, dx)
    gpu.avits_ckpt8_unpack(qo, so, dxo)
    assert torch.equal(dx[own], dxo)


def test_codes_past_two_to_the_31_bytes(gpu):
    import torch
    K, M, N = 2048, (1 << 21) + 21, 8
    x = _randn(M, K)
    q = torch.empty(M, K // 2, dtype=torch.uint8, device="cuda")
    s = torch.empty(*gpu.avits_mxfp4_scale_shape(M, K), dtype=torch.uint8, device="cuda")
    gpu.avits_mxfp4_quantize(x, q, s)
    codes, e = oracle.hold(_np(x[-21:]), 4)
    qo, so = oracle.mx_pack(codes, e)
    assert np.array_equal(q[-21:].cpu().numpy(), qo) and np.array_equal(s[:, M - 21:M].cpu().numpy(), so[:, :21])
    gpu.avits_mxfp4_dequantize(q, s, x)
    xv = oracle.held_values(codes, e, 4)
    assert np.array_equal(_np(x[-21:]), xv)
    wq, ws, w = _held(np.random.default_rng(0), N, K)
    out = torch.empty(M, N, device="cuda")
    gpu.avits_mxfp4_linear(q, s, wq, ws, None, out)
    # Sums of K exact products over K / 128 instructions and a few joins.
    assert_within(_np(out[-21:]), xv @ w.T, 2.0 ** -23 * (K / 128 + 9) * (np.abs(xv) @ np.abs(w).T))


def test_outputs_past_two_to_the_31_elements(gpu):
    import torch
    M, N, K = (1 << 20) + 21, 2056, 32
    rng = np.random.default_rng(1)
    wq, ws, w = _held(rng, N, K)
    x = _randn(M, K)
    q = torch.empty(M, K // 2, dtype=torch.uint8, device="cuda")
    s = torch.empty(*gpu.avits_mxfp4_scale_shape(M, K), dtype=torch.uint8, device="cuda")
    gpu.avits_mxfp4_quantize(x, q, s)
    res, gate = _randn(M, N), _randn(2, N)
    off = [0, M - 9, M]
    out = torch.empty_like(res)
    gpu.avits_mxfp4_linear(q, s, wq, ws, None, out, gate=gate, resid=res, off=off)
    codes, e = oracle.hold(_np(x[-21:]), 4)
    xv = oracle.held_values(codes, e, 4)
    g = _np(gate)[[0] * 12 + [1] * 9]
    ref, size = _np(res[-21:]) + g * (xv @ w.T), np.abs(xv) @ np.abs(w).T
    tol = np.abs(g) * 2.0 ** -23 * (K / 128 + 10) * size + 2.0 ** -23 * np.abs(ref)
    assert_within(_np(out[-21:]), ref, tol + 2.0 ** -8 * (np.abs(ref) + tol))
    # The gradient: dx [M, 2080] from a weight of 8 rows.
    wq, ws, w = _held(rng, 8, 2080)
    dy, dx = _randn(M, 8), torch.empty(M, 2080, dtype=torch.bfloat16, device="cuda")
    del out, res
    gpu.avits_mxfp4_linear_backward(dy, wq, ws, dx)
    d = _np(dy[-21:])
    ref, err = d @ w, 2.0 ** -23 * 9 * (np.abs(d) @ np.abs(w))
    assert_within(_np(dx[-21:]), ref, err + 2.0 ** -8 * (np.abs(ref) + err))


SPLIT = (1030, 1032, 4128)     # its contraction is split, so it needs a workspace


def test_a_workspace_made_by_the_call_belongs_to_its_stream(gpu):
    """Memory that the current stream gets right after the call is not the
    workspace of work that another stream has not done yet."""
    import torch
    M, N, K = SPLIT
    rng = np.random.default_rng(2)
    xq, xs, _ = _held(rng, M, K)
    wq, ws, _ = _held(rng, N, K)
    need = gpu.avits_mxfp4_linear_workspace_bytes(M, N, K)
    assert need > 0
    want = torch.empty(M, N, device="cuda")
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for handle in (side, side.cuda_stream):
        busy = torch.ones(4096, 4096, device="cuda")
        out = torch.empty_like(want)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(20):
                busy = busy @ busy * 2.0 ** -12     # keeps the stream behind the current one
        gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, out, stream=handle)
        junk = [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        del junk
    out = torch.empty_like(want)
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, out, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_graphs_that_share_a_workspace(gpu):
    """Two captured products and a captured gradient over one workspace,
    replayed in turn with eager calls between."""
    import torch
    M, N, K = SPLIT
    rng = np.random.default_rng(3)
    wq, ws, _ = _held(rng, N, K)
    pairs = [_held(rng, M, K)[:2] for _ in range(2)]
    dy, dx = _randn(70, N), torch.empty(70, K, dtype=torch.bfloat16, device="cuda")
    outs = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    work = torch.empty(max(gpu.avits_mxfp4_linear_workspace_bytes(M, N, K),
                           gpu.avits_mxfp4_linear_backward_workspace_bytes(70, N, K, 1)), dtype=torch.uint8, device="cuda")
    calls = [lambda i=i: gpu.avits_mxfp4_linear(*pairs[i], wq, ws, None, outs[i], workspace=work) for i in range(2)]
    calls.append(lambda: gpu.avits_mxfp4_linear_backward(dy, wq, ws, dx, workspace=work))
    results = outs + [dx]
    want = []
    for call, t in zip(calls, results):
        call()
        want.append(t.clone())
    graphs = []
    for call in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()
    for turn in range(4):
        for k in ((0, 1, 2), (2, 1, 0))[turn % 2]:
            results[k].zero_()
            graphs[k].replay()
            calls[(k + 1) % 3]()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, results)), turn


def test_a_workspace_on_the_host_is_refused(gpu):
    import torch
    M, N, K = SPLIT
    rng = np.random.default_rng(4)
    xq, xs, _ = _held(rng, 8, K)
    wq, ws, _ = _held(rng, 16, K)
    with pytest.raises(gpu.AvitsError):
        gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, torch.empty(8, 16, device="cuda"), workspace=torch.empty(64, dtype=torch.uint8))
    with pytest.raises(gpu.AvitsError):
        gpu.avits_mxfp4_linear(xq, xs, wq, ws, torch.zeros(16), torch.empty(8, 16, device="cuda"))

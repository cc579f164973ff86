"""4-bit products whose workgroups take several tiles, the longest rows and
contractions that are allowed, sixteen images, and calls on two streams at once."""
import pytest

from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _held(gpu, M, K, seed):
    """Random codes and scales, anything in the scales' padding rows, and the values as float64."""
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    q = torch.randint(0, 256, (M, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.randint(124, 131, gpu.avits_mxfp4_scale_shape(M, K), generator=g, device="cuda", dtype=torch.uint8)
    if K % 64:
        s[-1, :, 1] = 0
    v = torch.empty(M, K, device="cuda")
    gpu.avits_mxfp4_dequantize(q, s, v)
    s[:, M:] = 255
    return q, s, v


def _rand(seed, *shape):
    import torch
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def _assert(got, ref, tol):
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), tuple(bad.nonzero()[0].tolist()))


def _sum_error(K, size):
    """Exact products in a chain of K / 128 instructions and a few joins, each within 2^-23 of what it adds."""
    return 2.0 ** -23 * (K / 128 + 9) * size


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(4200, 4104, 256), (4200, 4104, 544), (4200, 4099, 768), (8300, 2051, 1056), (2100, 8200, 2080),
                                   (33000, 515, 96), (70000, 300, 288), (300, 70000, 288)])
def test_several_tiles_to_a_workgroup(gpu, M, N, K, dtype):
    """More than 256 tiles, of one step and of several, with rows of whole 16-byte chunks and without."""
    import torch
    (xq, xs, x), (wq, ws, w) = _held(gpu, M, K, M), _held(gpu, N, K, N)
    dt = TORCH_DT[dtype]
    b, res, gate = _rand(1, N).to(dt), _rand(2, M, N).to(dt), _rand(3, 3, N).to(dt)
    prod, size = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
    err = _sum_error(K, size)
    del size
    out = torch.full((M + 1, N), 7.0, dtype=dt, device="cuda")
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, b, out[:M])
    ref = prod + b.double()
    _assert(out[:M], ref, err + 2.0 ** -23 * ref.abs() + HALF[dtype] * (ref.abs() + err))
    assert (out[M] == 7.0).all()
    bare = torch.empty(M, N, dtype=dt, device="cuda")
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, bare)
    _assert(bare, prod, err + HALF[dtype] * (prod.abs() + err))
    off = [0, M // 3 + 1, M // 3 + 1, M]      # the second image has no rows
    y = torch.full((M + 1, N), 7.0, dtype=dt, device="cuda")
    y[:M] = res
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, b, y[:M], gate=gate, resid=y[:M], off=off)
    g = torch.cat([gate[:1].expand(off[1], N), gate[2:].expand(M - off[1], N)]).double()
    want = res.double() + g * ref
    tol = g.abs() * (err + 2.0 ** -22 * ref.abs()) + 2.0 ** -23 * want.abs()
    _assert(y[:M], want, tol + HALF[dtype] * (want.abs() + tol))
    assert (y[M] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [2, 300])
@pytest.mark.parametrize("N", [(1 << 21) - 1, (1 << 21) - 8])
def test_the_most_outputs(gpu, M, N, dtype):
    import torch
    K, dt = 32, TORCH_DT[dtype]
    (xq, xs, x), (wq, ws, w) = _held(gpu, M, K, M), _held(gpu, N, K, 5)
    b = _rand(1, N).to(dt)
    out = torch.full((M + 1, N), 7.0, dtype=dt, device="cuda")
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, b, out[:M])
    for lo in (0, (1 << 20) - 300, N - 700):
        c = slice(lo, min(lo + 700, N))
        ref, size = x.double() @ w[c].double().t() + b[c].double(), x.double().abs() @ w[c].double().abs().t()
        tol = _sum_error(K, size) + 2.0 ** -23 * ref.abs()
        _assert(out[:M, c], ref, tol + HALF[dtype] * (ref.abs() + tol))
    assert (out[M] == 7.0).all()
    del out
    # The gradient sums over them all: of dy's few columns that are not 0, at both ends.
    dy = torch.zeros(M, N, dtype=dt, device="cuda")
    at = torch.tensor([0, 1, 31, 8191, (1 << 20) + 5, N - 9, N - 2, N - 1], device="cuda")
    dy[:, at] = _rand(4, M, len(at)).to(dt)
    dx = torch.full((M + 1, K), 7.0, dtype=dt, device="cuda")
    gpu.avits_mxfp4_linear_backward(dy, wq, ws, dx[:M])
    d, wa = dy[:, at].double(), w[at].double()
    ref, tol = d @ wa, 2.0 ** -23 * 32 * (d.abs() @ wa.abs())     # at most eight terms, three parts of each, and a few joins
    _assert(dx[:M], ref, tol + HALF[dtype] * (ref.abs() + tol))
    assert (dx[M] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N", [(2, 3), (300, 260)])
def test_the_longest_contraction(gpu, M, N, dtype):
    import torch
    K, dt = (1 << 21) - 32, TORCH_DT[dtype]
    (xq, xs, x), (wq, ws, w) = _held(gpu, M, K, M), _held(gpu, N, K, 7)
    # One nonzero block in eight thousand, at both ends among them, so that sums are short and exact.
    keep = torch.zeros(K // 32, dtype=torch.bool, device="cuda")
    keep[torch.tensor([0, 1, 7, 8, 8191, 32768, K // 32 - 2, K // 32 - 1], device="cuda")] = True
    mask = keep.repeat_interleave(32)
    xq.view(M, K // 32, 16)[:, ~keep] = 0
    xv, wv = x[:, mask].double(), w[:, mask].double()
    out = torch.full((M + 1, N), 7.0, dtype=dt, device="cuda")
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, out[:M])
    ref, tol = xv @ wv.t(), _sum_error(256, xv.abs() @ wv.abs().t())
    _assert(out[:M], ref, tol + HALF[dtype] * (ref.abs() + tol))
    assert (out[M] == 7.0).all()
    dy = _rand(3, M, N).to(dt)
    dx = torch.full((M + 1, K), 7.0, dtype=dt, device="cuda")
    gpu.avits_mxfp4_linear_backward(dy, wq, ws, dx[:M])
    ref, size = dy.double() @ wv, dy.double().abs() @ wv.abs()
    tol = 2.0 ** -23 * (3 * N / 32 + 9) * size
    _assert(dx[:M, mask], ref, tol + HALF[dtype] * (ref.abs() + tol))
    assert (dx[M] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(5, 300, 96), (1700, 2056, 4128), (1700, 1031, 4128), (4300, 4104, 288)])
def test_sixteen_images(gpu, M, N, K, dtype):
    """Each row takes its image's gate: the rows of every image as in a call of their own gate."""
    import torch
    (xq, xs, _), (wq, ws, _) = _held(gpu, M, K, M), _held(gpu, N, K, N)
    dt = TORCH_DT[dtype]
    res, mod = _rand(2, M, N).to(dt), _rand(3, 16, 6, N).to(dt)
    gate = mod[:, 5]
    cut = torch.randint(0, M + 1, (15,), generator=torch.Generator().manual_seed(M)).sort().values.tolist()
    off = [0] + cut + [M]
    out, one = torch.empty(M, N, dtype=dt, device="cuda"), torch.empty(M, N, dtype=dt, device="cuda")
    gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, out, gate=gate, resid=res, off=off)
    for i in range(16):
        gpu.avits_mxfp4_linear(xq, xs, wq, ws, None, one, gate=gate[i].contiguous(), resid=res)
        assert torch.equal(out[off[i]:off[i + 1]], one[off[i]:off[i + 1]]), i


def test_two_streams_at_once(gpu):
    """Products in parts and gradients on two streams, each with its own workspace: the same bits as alone."""
    import torch
    M, N, K = 1030, 1032, 4128
    (wq, ws, _) = _held(gpu, N, K, 1)
    xs = [_held(gpu, M, K, 2 + i)[:2] for i in range(2)]
    dy = [_rand(9 + i, 70, N).bfloat16() for i in range(2)]
    out = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    dx = [torch.empty(70, K, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    need = max(gpu.avits_mxfp4_linear_workspace_bytes(M, N, K), gpu.avits_mxfp4_linear_backward_workspace_bytes(70, N, K, 1))
    work = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def both(i, stream):
        gpu.avits_mxfp4_linear(*xs[i], wq, ws, None, out[i], workspace=work[i], stream=stream)
        gpu.avits_mxfp4_linear_backward(dy[i], wq, ws, dx[i], workspace=work[i], stream=stream)

    for i in range(2):
        both(i, None)
    want = [t.clone() for t in out + dx]
    for t in out + dx:
        t.fill_(3.0)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            both(i, streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, out + dx))

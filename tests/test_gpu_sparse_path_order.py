"""SparseAttention's calls in other orders than forward, backward."""
import pytest

from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu


def _path(H, Hk, d, rows, dtype, seed, **kw):
    import torch
    from paper_2608_17995_amd.step import SparseAttention
    g = torch.Generator().manual_seed(seed)
    dt = TORCH_DT[dtype]
    gains = [(1 + 0.3 * torch.randn(d, generator=g)).to(dt).cuda() for _ in range(2)]
    kw = {**dict(dims=(8, 28, 28) if d == 64 else (16, 56, 56), keep=2, lead=64, batch=2), **kw}
    path = SparseAttention(rows, H, d, Hk=Hk, g_q=gains[0], g_k=gains[1], dtype=dt, **kw)

    def rows_of(n):
        qkv = torch.randn(n, (H + 2 * Hk) * d, generator=g).to(dt).cuda()
        pos = torch.randint(0, 40, (n, 3), generator=g, dtype=torch.int32).cuda()
        dout = torch.randn(n, H, d, generator=g).to(dt).cuda()
        return dict(qkv=qkv, pos=pos, dout=dout, out=torch.full_like(dout, 5.0), dqkv=torch.full_like(qkv, 5.0),
                    dg=[torch.full((d,), 5.0, device="cuda") for _ in range(2)])
    return path, rows_of


def _forward(path, r, **kw):
    path.forward(r["qkv"], r["pos"], r["out"], **kw)


def _backward(path, r):
    path.backward(r["dout"], r["qkv"], r["pos"], r["out"], r["dqkv"], *r["dg"])


# What the run in between takes: other rows, more, fewer, packed otherwise, none.
@pytest.mark.parametrize("n,off", [(900, None), (900, (0, 400, 820)), (130, (0, 1, 130)), (1, None), (0, None)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d", [(4, 2, 64), (2, 2, 128)])
def test_run_between(gpu, H, Hk, d, dtype, n, off):
    """forward, run on other rows, backward: the gradients of the forward's rows, and run's output as an object of its own gives it."""
    import torch
    path, rows_of = _path(H, Hk, d, 900, dtype, seed=21, tune=True)
    a, b = rows_of(850), rows_of(n)
    _forward(path, a, off=(0, 333, 850), pos_scale=0.5)
    _backward(path, a)
    want = [t.clone() for t in (a["out"], a["dqkv"], *a["dg"])]
    for t in (a["out"], a["dqkv"], *a["dg"]):
        t.fill_(5)
    plain, _ = _path(H, Hk, d, 900, dtype, seed=21)
    alone = plain.run(b["qkv"], b["pos"], b["out"].clone(), off=off)
    _forward(path, a, off=(0, 333, 850), pos_scale=0.5)
    path.run(b["qkv"], b["pos"], b["out"], off=off)
    _backward(path, a)
    assert all(torch.equal(x, y) for x, y in zip((a["out"], a["dqkv"], *a["dg"]), want))
    assert torch.equal(b["out"], alone)


def test_runs_between_in_a_graph(gpu):
    """A captured run replayed between an eager forward and its backward, and the other way round."""
    import torch
    path, rows_of = _path(4, 4, 64, 700, "bf16", seed=23, tune=True)
    a, b = rows_of(700), rows_of(513)
    _forward(path, a)
    _backward(path, a)
    path.run(b["qkv"], b["pos"], b["out"])
    want = [t.clone() for t in (a["out"], a["dqkv"], *a["dg"], b["out"])]
    run, tune = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(run):
        path.run(b["qkv"], b["pos"], b["out"])
    with torch.cuda.graph(tune):
        _forward(path, a)
        path.run(b["qkv"], b["pos"], b["out"])
        _backward(path, a)
    for _ in range(3):
        for t in (a["out"], a["dqkv"], *a["dg"], b["out"]):
            t.fill_(5)
        _forward(path, a)
        run.replay()
        _backward(path, a)
        assert all(torch.equal(x, y) for x, y in zip((a["out"], a["dqkv"], *a["dg"], b["out"]), want))
        for t in (a["out"], a["dqkv"], *a["dg"], b["out"]):
            t.fill_(5)
        tune.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((a["out"], a["dqkv"], *a["dg"], b["out"]), want))

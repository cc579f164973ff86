"""Mxfp4Mlp made on one stream and used on another."""
import pytest

from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu


def _weights(D, F, dtype, seed=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(TORCH_DT[dtype]).cuda()  # noqa: E731
    return (r(F, D, std=D ** -0.5), r(F, std=0.1), r(D, F, std=F ** -0.5), r(D, std=0.1)), r(77, D), r(6, D, std=0.3)


def _keep_busy():
    """Work that keeps the current stream going for some ten milliseconds."""
    import torch
    busy = torch.ones(4096, 4096, device="cuda")
    for _ in range(40):
        busy = busy @ busy * 2.0 ** -12


def test_the_weights_are_held_when_the_constructor_returns(gpu):
    import torch
    from paper_2608_17995_amd.step import Mxfp4Mlp
    w, _, _ = _weights(256, 512, "bf16")
    torch.cuda.synchronize()
    _keep_busy()
    assert not torch.cuda.current_stream().query()
    Mxfp4Mlp(*w, rows=80, tune=True)
    assert torch.cuda.current_stream().query()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_calls_on_another_stream(gpu, dtype):
    """Without a wait of the caller's, behind queued work of the constructor's stream: the bits of an
    object made and used in order."""
    import torch
    from paper_2608_17995_amd.step import Mxfp4Mlp
    w, x, mod = _weights(256, 512, dtype)
    z, dx, out = (torch.empty_like(x) for _ in range(3))
    ds = torch.empty(256, device="cuda")

    def step(mlp, stream):
        mlp.forward(x, mod[3], mod[4], z, stream=stream)
        mlp.backward(x, mod[4], dx, ds, stream=stream)
        mlp.run(x, mod[3], mod[4], mod[5], out, stream=stream)

    step(Mxfp4Mlp(*w, rows=80, tune=True), None)
    torch.cuda.synchronize()
    want = [t.clone() for t in (z, dx, ds, out)]
    side = torch.cuda.Stream()
    for t in (z, dx, ds, out):
        t.fill_(3.0)
    torch.cuda.synchronize()
    _keep_busy()
    mlp = Mxfp4Mlp(*w, rows=80, tune=True)
    step(mlp, side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (z, dx, ds, out)))


def test_made_within_a_capture(gpu):
    """The weights are quantised by every replay then, from what they hold at that time."""
    import torch
    from paper_2608_17995_amd.step import Mxfp4Mlp
    w, x, mod = _weights(64, 128, "bf16")
    out, want = torch.empty_like(x), torch.empty_like(x)
    Mxfp4Mlp(*w, rows=80).run(x, mod[3], mod[4], mod[5], out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mlp = Mxfp4Mlp(*w, rows=80)
        mlp.run(x, mod[3], mod[4], mod[5], out)
    for k in range(3):
        w[0].mul_(-1.5)
        Mxfp4Mlp(*w, rows=80).run(x, mod[3], mod[4], mod[5], want)
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), k

"""The blocks' means and the choice of key blocks against the oracle: bit for bit."""
import numpy as np
import pytest

import oracle
from _gpu import TORCH_DT

pytestmark = pytest.mark.gpu


def _rows(M, H, d, dtype, g, extra=0):
    import torch
    return torch.randn(M, H + extra, d, generator=g).to(TORCH_DT[dtype]).cuda()[:, :H]


def _means(gpu, x, size, off):
    import torch
    n = len(oracle.cut(off, size))
    out = torch.full((n, x.shape[1], x.shape[2]), 7.0, dtype=torch.float64, device="cuda")
    gpu.avits_block_means(x, size, out, off=off)
    want = oracle.block_means(x.double().cpu().numpy(), off, size)
    got = out.cpu().numpy()
    # A sum of `size` terms in 64 bits, and a division.
    bound = (size + 1) * 2.0 ** -53 * oracle.block_means(np.abs(x.double().cpu().numpy()), off, size)
    assert (np.abs(got - want) <= bound).all()
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d,q_off,k_off,q_lead,k_lead,keep", [
    (1, 1, 64, (0, 1), (0, 1), 0, 0, 1), (4, 4, 64, (0, 701), (0, 701), 77, 77, 3), (6, 2, 128, (0, 333), (0, 333), 0, 0, 0),
    (4, 1, 64, (0, 1), (0, 5000), 0, 100, 9), (8, 8, 128, (0, 300, 300, 777), (0, 300, 300, 777), 40, 40, 2),
    (2, 2, 64, (0, 5, 9), (0, 0, 700), 0, 0, 4), (2, 1, 64, (0, 2300), (0, 4200), 0, 64, 30), (3, 3, 64, (0, 257), (0, 130), 0, 0, 50),
    (5, 5, 64, tuple(range(0, 161, 10)), tuple(range(0, 1601, 100)), 0, 1, 1)])
def test_choice(gpu, H, Hk, d, q_off, k_off, q_lead, k_lead, keep, dtype):
    import torch
    g = torch.Generator().manual_seed(1)
    q, k = _rows(q_off[-1] + 3, H, d, dtype, g, 2 * Hk), _rows(k_off[-1] + 5, Hk, d, dtype, g, 1)
    qm, km = _means(gpu, q, 128, q_off), _means(gpu, k, 64, k_off)
    want = oracle.block_select(qm.cpu().numpy(), km.cpu().numpy(), keep, q_off, k_off, q_lead, k_lead)
    for words in (-(-want.shape[2] // 64), -(-want.shape[2] // 64) + 2):
        mask = torch.full((H, want.shape[1], words), -1, dtype=torch.int64, device="cuda")
        gpu.avits_block_select(qm, km, keep, mask, q_lead=q_lead, k_lead=k_lead, q_off=q_off, k_off=k_off)
        assert np.array_equal(mask.cpu().numpy(), oracle.words(want, words))


@pytest.mark.parametrize("nk,keep", [(1100, 40), (4097, 1), (16384, 700)])
def test_long_sequences(gpu, nk, keep):
    """More key blocks than 16 rows' scores have room for."""
    import torch
    g = torch.Generator().manual_seed(2)
    qm = torch.randn(19, 2, 64, generator=g, dtype=torch.float64).cuda()
    km = torch.randn(nk, 1, 64, generator=g, dtype=torch.float64).cuda()
    mask = torch.full((2, 19, -(-nk // 64)), -1, dtype=torch.int64, device="cuda")
    gpu.avits_block_select(qm, km, keep, mask, k_lead=100)
    want = oracle.block_select(qm.cpu().numpy(), km.cpu().numpy(), keep, (0, 19 * 128), (0, 64 * nk), 0, 100)
    assert np.array_equal(mask.cpu().numpy(), oracle.words(want))


def test_ties_and_bad_values(gpu):
    """Equal scores: the lowest block; -0 equals +0; NaN last; infinities in order."""
    import torch
    qm = torch.zeros(3, 1, 64, dtype=torch.float64, device="cuda")
    km = torch.zeros(200, 1, 64, dtype=torch.float64, device="cuda")
    qm[:, 0, 0] = torch.tensor([1.0, -1.0, 0.0])
    km[:, 0, 0] = torch.tensor([float(i % 5 - 2) for i in range(200)])
    km[7, 0, 0], km[11, 0, 0], km[13, 0, 0] = float("inf"), float("nan"), -float("inf")
    km[20:30, 0, 0] = -0.0
    for keep in (0, 1, 5, 39, 80, 81, 150, 196, 197, 198, 199, 200, 300):
        mask = torch.empty(3, 1, 4, dtype=torch.int64, device="cuda").view(1, 3, 4)
        gpu.avits_block_select(qm, km, keep, mask)
        with np.errstate(invalid="ignore"):
            want = oracle.block_select(qm.cpu().numpy(), km.cpu().numpy(), keep, (0, 384), (0, 12800))
        assert np.array_equal(mask.cpu().numpy(), oracle.words(want)), keep


def test_other_stream_and_graph(gpu):
    import torch
    g = torch.Generator().manual_seed(4)
    x = _rows(2000, 8, 64, "bf16", g)
    off = (0, 900, 2000)
    qm, km = (torch.empty(len(oracle.cut(off, n)), 8, 64, dtype=torch.float64, device="cuda") for n in (128, 64))
    mask = torch.empty(8, qm.shape[0], 1, dtype=torch.int64, device="cuda")

    def run(**kw):
        gpu.avits_block_means(x, 128, qm, off=off, **kw)
        gpu.avits_block_means(x, 64, km, off=off, **kw)
        gpu.avits_block_select(qm, km, 5, mask, q_lead=70, k_lead=70, q_off=off, k_off=off, **kw)
    run()
    want = mask.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    mask.zero_()
    torch.cuda.synchronize()
    run(stream=side)
    side.synchronize()
    assert torch.equal(mask, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        mask.zero_()
        km.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(mask, want)

"""The attention half's calls of so many rows that their workgroups have more than 2^32 threads together.  One head, so that
the rows fit the card."""
import pytest

pytestmark = pytest.mark.gpu


def _room(gib):
    import torch
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip(f"needs {gib} GiB of device memory")


def test_backward_of_2_26_rows(gpu):
    """A few of 2^19 query blocks keep a key: the same bits as a call of these blocks alone; the others' dq is zero."""
    import torch
    _room(45)
    blocks = torch.tensor([0, 3, 70000, (1 << 19) - 1, 1 << 19])
    M, N, bf16 = (1 << 26) + 100, 70, torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda n: torch.randn(n, 1, 64, generator=g, device="cuda").to(bf16)  # noqa: E731
    small = {n: normal(4 * 128 + 100) for n in ("q", "do")}
    k, v = normal(N), normal(N)
    nq = (M + 127) // 128
    assert nq == (1 << 19) + 1
    rows = (blocks[:, None] * 128 + torch.arange(128)).flatten()[:4 * 128 + 100].cuda()
    large = {n: torch.zeros(M, 1, 64, dtype=bf16, device="cuda").index_copy_(0, rows, t) for n, t in small.items()}
    mask = torch.zeros(1, nq, 1, dtype=torch.int64, device="cuda")
    mask[0, blocks.cuda(), 0] = 3
    out = []
    for t, m in ((small, None), (large, mask)):
        n = len(t["q"])
        o, dq = (torch.full((n, 1, 64), 5.0, dtype=bf16, device="cuda") for _ in range(2))
        lse, dk, dv = torch.empty(1, n, device="cuda"), torch.empty_like(k), torch.empty_like(v)
        gpu.avits_sparse_attention(t["q"], k, v, o, m, lse)
        gpu.avits_sparse_attention_backward(t["do"], t["q"], k, v, o, lse, dq, dk, dv, m)
        out.append((o, dq, dk, dv))
    (o, dq, dk, dv), (lo, ldq, ldk, ldv) = out
    assert torch.equal(dk, ldk) and torch.equal(dv, ldv) and dk.any()
    assert torch.equal(lo[rows], o) and torch.equal(ldq[rows], dq) and dq.any()
    for t in (lo, ldq):
        t[rows] = 0
        assert not t.any()


def test_means_of_2_30_rows(gpu):
    import torch
    _room(160)
    M = (1 << 30) + 100
    x = torch.ones(M, 1, 64, dtype=torch.bfloat16, device="cuda")
    x[:64] = 2
    x[-36:] = 3           # the last block's rows
    n = (M + 63) // 64
    means = torch.full((n, 1, 64), 5.0, dtype=torch.float64, device="cuda")
    gpu.avits_block_means(x, 64, means)
    assert n == (1 << 24) + 2
    assert (means[0] == 2).all() and (means[-1] == 3).all() and (means[1:-1] == 1).all()


def test_choice_for_2_23_query_blocks(gpu):
    """More key blocks than two query blocks' scores have room for: a workgroup to each query block."""
    import torch
    _room(25)
    nq, nk = (1 << 23) + 3, 8193
    g = torch.Generator(device="cuda").manual_seed(2)
    qm = torch.randn(nq, 1, 64, generator=g, device="cuda", dtype=torch.float32).double()
    km = torch.randn(nk, 1, 64, generator=g, device="cuda", dtype=torch.float32).double()
    mask = torch.full((1, nq, 129), 5, dtype=torch.int64, device="cuda")
    gpu.avits_block_select(qm, km, 1, mask)
    at = torch.cat([torch.arange(50), torch.arange(nq - 50, nq), torch.randint(0, nq, (200,))]).cuda()
    best = (qm[at, 0] @ km[:, 0].t().contiguous()).argmax(1)
    want = torch.zeros(len(at), 129, dtype=torch.int64, device="cuda")
    want[torch.arange(len(at), device="cuda"), best // 64] = 1 << best % 64
    assert torch.equal(mask[0, at], want)
    # One bit in every row.
    assert ((mask[0] != 0).sum(1) == 1).all() and ((mask[0] & (mask[0] - 1)) == 0).all()

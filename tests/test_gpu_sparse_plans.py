"""Sparse attention where its work is shared out differently: many and few units, lists of uneven lengths, workspaces of
exactly the size, rows far apart, two calls at once, tensors that do not fit together."""
import numpy as np
import pytest

import oracle
from _gpu import TORCH_DT
from _sparse import backward, check_backward, check_forward, forward, make

pytestmark = pytest.mark.gpu


def _uneven(s, text, seed):
    """The first `text` query blocks keep everything, one none, the others key block 0 and a few more."""
    import torch
    rng = np.random.default_rng(seed)
    on = s["on"]
    on[:] = rng.random(on.shape) < 0.12
    on[:, :, 0] = True
    on[:, :text] = True
    on[:, text] = False
    s["mask"].copy_(torch.from_numpy(oracle.words(on, s["mask"].shape[-1]).copy()))
    return s


def _heads(s, lo, hi):
    """The tensors of key heads lo .. hi - 1 and their query heads."""
    g = s["q"].shape[1] // s["k"].shape[1]
    part = dict(s, on=s["on"][lo * g:hi * g], lse=s["lse"][lo * g:hi * g])
    for n in ("q", "o", "do", "dq"):
        part[n] = s[n][:, lo * g:hi * g]
    for n in ("k", "v", "dk", "dv"):
        part[n] = s[n][:, lo:hi]
    return part


def _both(gpu, s, parts=None, **kw):
    forward(gpu, s, **kw)
    backward(gpu, s, **kw)
    on = None if kw.get("mask", 0) is None else "mask"
    for p in [s] if parts is None else [_heads(s, *r) for r in parts]:
        check_forward(p, on)
        check_backward(p, on)


# Blocks x heads: 96 and 192; 45 and 5 x 45, keys and queries apart; 288 with grouped keys; packed.
@pytest.mark.parametrize("H,Hk,d,q_off,k_off", [
    (8, 8, 128, (0, 1500), (0, 1500)), (45, 5, 64, (0, 100), (0, 2900)), (9, 3, 64, (0, 4000), (0, 300)),
    (16, 4, 64, (0, 1, 900, 900, 2100), (0, 70, 1000, 1100, 1164))])
def test_uneven_lists(gpu, H, Hk, d, q_off, k_off):
    s = make(H, Hk, d, q_off, k_off, "bf16", seed=31)
    _both(gpu, _uneven(s, min(2, s["on"].shape[1] - 1), 31))


def test_many_units(gpu):
    """More query blocks than a plan is made for (2560; keys' 4608)."""
    s = make(512, 512, 64, (0, 520), (0, 520), "bf16", seed=33)
    _both(gpu, s, [(0, 3), (255, 257), (510, 512)])


def test_long_lists_of_pairs(gpu):
    """1088 (head, query block) pairs to a key block, more than are looked at together."""
    s = make(64, 1, 64, (0, 2100), (0, 200), "bf16", seed=35, density=0.8)
    _both(gpu, s)
    s["mask"].fill_(-1)
    _both(gpu, dict(s, on=np.ones_like(s["on"])))


@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("H,Hk,d,M,N", [(1, 1, 128, 3000, 3000), (4, 1, 64, 130, 4500), (2, 2, 128, 4100, 100)])
def test_few_units(gpu, H, Hk, d, M, N, dense):
    s = make(H, Hk, d, (0, M), (0, N), "bf16", seed=37)
    _both(gpu, s, **(dict(mask=None) if dense else {}))


@pytest.mark.parametrize("H,Hk,d,M,N", [(16, 16, 64, 1100, 1100), (12, 4, 128, 1500, 700), (40, 40, 64, 70, 500)])
def test_fp32_rows(gpu, H, Hk, d, M, N):
    """Workgroups of 64 rows and of 16, on either side."""
    _both(gpu, make(H, Hk, d, (0, M), (0, N), "f32", seed=39))


@pytest.mark.parametrize("H,Hk,M,N,dense", [(8, 8, 1500, 1500, False), (1, 1, 900, 2500, True), (2, 1, 1, 5000, False), (4, 4, 300, 300, False)])
def test_workspace_of_the_size(gpu, H, Hk, M, N, dense):
    """Nothing behind it is written; one byte less is refused; one made for more rows will do."""
    import torch
    s = make(H, Hk, 128, (0, M), (0, N), "bf16", seed=41, extra=0)
    kw = dict(mask=None) if dense else {}
    need = (gpu.avits_sparse_attention_workspace_bytes(M, N, 1, H, 128, gpu.BF16),
            gpu.avits_sparse_attention_backward_workspace_bytes(M, N, 1, H, Hk, 128, gpu.BF16))
    for call, n, check in ((forward, need[0], check_forward), (backward, need[1], check_backward)):
        buf = torch.full((n + 4096,), 171, dtype=torch.uint8, device="cuda")
        call(gpu, s, workspace=buf[:n], **kw)
        assert (buf[n:] == 171).all()
        check(s, None if dense else "mask")
    first = [s[n].clone() for n in ("o", "dq", "dk", "dv")]
    with pytest.raises(gpu.AvitsError):
        backward(gpu, s, workspace=buf[:need[1] - 1], **kw)
    large = torch.empty(max(gpu.avits_sparse_attention_workspace_bytes(9000, 9000, 4, H, 128, gpu.BF16),
                            gpu.avits_sparse_attention_backward_workspace_bytes(9000, 9000, 4, H, Hk, 128, gpu.BF16)),
                        dtype=torch.uint8, device="cuda")
    forward(gpu, s, workspace=large, **kw)
    backward(gpu, s, workspace=large, **kw)
    assert all(torch.equal(s[n], t) for n, t in zip(("o", "dq", "dk", "dv"), first))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_apart(gpu, dtype):
    """Row strides of 2^23 elements and more than 2^31 of them in all: the same bits as from rows side by side."""
    import torch
    H, Hk, d, M = 2, 1, 64, 300
    s = make(H, Hk, d, (0, M), (0, M), dtype, seed=43, extra=0, packed=False)
    forward(gpu, s)
    backward(gpu, s)
    dt = TORCH_DT[dtype]
    far = torch.empty(M, 1 << 23, dtype=dt, device="cuda")
    at, wide = 0, dict(s)
    for n, heads in (("q", H), ("k", Hk), ("v", Hk), ("do", H), ("o", H), ("dq", H), ("dk", Hk), ("dv", Hk)):
        wide[n] = far[:, at:at + heads * d].view(M, heads, d)
        wide[n].copy_(s[n]) if n in ("q", "k", "v", "do") else wide[n].fill_(5)
        at += heads * d
    forward(gpu, wide)
    backward(gpu, wide)
    for n in ("o", "dq", "dk", "dv"):
        assert torch.equal(wide[n], s[n]), n
    for n in ("q", "k"):
        kw = dict(pos=torch.arange(M, dtype=torch.int32, device="cuda"), freq=gpu.avits_rope_frequencies((d,)).cuda())
        want = torch.empty_like(s[n])
        gpu.avits_qk_norm_rope(s[n], None, want, None, **kw)
        gpu.avits_qk_norm_rope(wide[n], None, wide["d" + n], None, **kw)
        assert torch.equal(wide["d" + n], want)
        back = torch.empty_like(s[n])
        gpu.avits_qk_norm_rope_backward(s["d" + n], None, s[n], None, back, None, **kw)
        wide["d" + n].copy_(s["d" + n])
        gpu.avits_qk_norm_rope_backward(wide["d" + n], None, wide[n], None, wide["d" + n], None, **kw)
        assert torch.equal(wide["d" + n], back)
        heads = s[n].shape[1]
        means = [torch.empty(5, heads, d, dtype=torch.float64, device="cuda") for _ in range(2)]
        gpu.avits_block_means(s[n], 64, means[0])
        gpu.avits_block_means(wide[n], 64, means[1])
        assert torch.equal(*means)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,M,N", [(2, 300, 300), (1, 5, 3000)])
@pytest.mark.parametrize("sign", [1, -1])
def test_huge_equal_logits(gpu, H, M, N, sign, dtype):
    """All logits +-2^117 / 8: the mean of the values, whatever their size."""
    import torch
    s = make(H, H, 64, (0, M), (0, N), dtype, seed=49, extra=0, packed=False)
    s["q"].zero_()
    s["k"].zero_()
    s["q"][:, :, 0], s["k"][:, :, 0] = 2.0 ** 60, sign * 2.0 ** 57
    forward(gpu, s, mask=None)
    v = s["v"].double()
    # The probabilities are exactly 1: N additions and a division in fp32, then one rounding.
    tol = (N + 2) * 2.0 ** -24 * v.abs().mean(0) + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * v.mean(0).abs()
    assert ((s["o"].double() - v.mean(0)).abs() <= 1.01 * tol).all()
    assert ((s["lse"] / (sign * 2.0 ** 114) - 1).abs() < 2.0 ** -21).all()


@pytest.mark.parametrize("M", [3, 110, 700])
def test_keys_alike(gpu, M):
    """Keys that share more than they differ by: a row's ds add up to zero, and what the keys share does not reach dq."""
    import torch
    s = make(4, 2, 64, (0, M), (0, M), "bf16", seed=51, extra=0, packed=False)
    s["k"] = (s["k"].float() + 8 * torch.randn(1, 2, 64, generator=torch.Generator().manual_seed(52)).cuda()).to(torch.bfloat16)
    s["q"].mul_(0.25)
    forward(gpu, s, mask=None)
    backward(gpu, s, mask=None)
    check_backward(s, None)
    q, k, v, do, o, lse = (s[n].double() for n in ("q", "k", "v", "do", "o", "lse"))
    for h in range(4):
        j = h // 2
        x = q[:, h] @ k[:, j].T * s["scale"]
        p = torch.exp(x - lse[h][:, None])
        delta = (do[:, h] * o[:, h]).sum(1)[:, None]
        ds = p * (do[:, h] @ v[:, j].T - delta)
        want = s["scale"] * ds @ k[:, j]
        # ds to two parts of 8 bits, 2^-16; logits, dout . v and delta of 64 products in fp32, sums of M.
        es = 2.0 ** -24 * (66 * (q[:, h].abs() @ k[:, j].T.abs()) * s["scale"] + 4 * x.abs() + 4 * lse[h].abs()[:, None] + 6)
        eds = ds.abs() * (es + 2.0 ** -16 + (M / 4 + 24) * 2.0 ** -24) + p * 68 * 2.0 ** -24 * (
            do[:, h].abs() @ v[:, j].T.abs() + (do[:, h] * o[:, h]).abs().sum(1)[:, None])
        tol = s["scale"] * eds @ k[:, j].abs()
        err = (s["dq"][:, h].double() - want).abs()
        assert (err <= tol + 2.0 ** -8 * (want.abs() + tol)).all(), (h, float((err - tol - 2.0 ** -8 * want.abs()).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [2.0 ** -64, 2.0 ** -30, 1.0])
def test_scales(gpu, scale, dtype):
    s = make(2, 1, 64, (0, 200), (0, 300), dtype, seed=53)
    s["scale"] = scale
    forward(gpu, s, scale=scale)
    check_forward(s)
    backward(gpu, s, scale=scale)
    check_backward(s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sixteen_sequences(gpu, dtype):
    """The most that a call takes, some without queries, some without keys."""
    q = (0, 5, 5, 133, 200, 201, 300, 428, 428, 500, 629, 700, 700, 710, 800, 801, 930)
    k = (0, 64, 70, 70, 300, 301, 400, 529, 600, 600, 700, 765, 800, 864, 864, 900, 1100)
    _both(gpu, make(3, 1, 64, q, k, dtype, seed=55))


def test_two_at_once(gpu):
    """Two streams, a workspace each, many times over: the results of one after the other."""
    import torch
    parts = [make(8, 8, 128, (0, 1200), (0, 1200), "bf16", seed=s) for s in (45, 46)]
    for s in parts:
        forward(gpu, s)
        backward(gpu, s)
    want = [[s[n].clone() for n in ("o", "lse", "dq", "dk", "dv")] for s in parts]
    streams = [torch.cuda.Stream() for _ in parts]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for s, st in zip(parts, streams):
            forward(gpu, s, stream=st)
            backward(gpu, s, stream=st)
    for st in streams:
        st.synchronize()
    for s, w in zip(parts, want):
        for n, t in zip(("o", "lse", "dq", "dk", "dv"), w):
            assert torch.equal(s[n], t), n


def test_tensors_that_do_not_fit(gpu):
    import torch
    s = make(4, 2, 64, (0, 200), (0, 200), "bf16", seed=47, extra=0)
    errors = (ValueError, TypeError, gpu.AvitsError)
    for bad in (dict(k=s["k"].float()), dict(v=s["v"].cpu()), dict(q=s["q"].half()), dict(k=s["k"][:, :1]), dict(v=s["v"][:199]),
                dict(o=s["o"][:, :3]), dict(o=s["o"].transpose(1, 2)), dict(lse=s["lse"].double()), dict(lse=s["lse"][:, :199]),
                dict(mask=s["mask"].int()), dict(mask=s["mask"][:3]), dict(mask=s["mask"][:, :, :0]), dict(mask=s["mask"][:, :1]),
                dict(q=torch.zeros(200, 4, 96, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(errors):
            forward(gpu, {**s, **bad})
    forward(gpu, s)
    for bad in (dict(dq=s["dq"].float()), dict(dk=s["dk"][:, :1]), dict(do=s["do"][:199]), dict(lse=s["lse"][:3])):
        with pytest.raises(errors):
            backward(gpu, {**s, **bad})

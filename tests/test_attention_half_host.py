"""Refusals of the norm-and-rotation, block choice and sparse attention calls: every call
below fails on the host, before any device memory is touched (or has nothing to do)."""
import ctypes
import math

import numpy as np
import pytest

import paper_2608_17995_amd as avits
from paper_2608_17995_amd import _binding as B

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
FAKE = 0x1000  # never dereferenced
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return avits.load()


def arr(*v):
    return (ctypes.c_int64 * len(v))(*v)


def rope(pos=FAKE, freq=FAKE, pos_scale=1.0, layout=0, axes=3, dims=(8, 28, 28)):
    return ctypes.addressof(_KEEP.setdefault((pos, freq, pos_scale, layout, axes, dims),
                                             B._Rope(pos, freq, pos_scale, layout, axes, (ctypes.c_int32 * 4)(*dims))))


_KEEP = {}
BAD_ROPES = [dict(axes=0), dict(axes=5), dict(layout=2), dict(dims=(8, 28, 30)), dict(dims=(7, 28, 28)), dict(dims=(-2, 28, 28)),
             dict(pos=None), dict(freq=None), dict(pos=FAKE + 2), dict(freq=FAKE + 4), dict(pos_scale=math.nan),
             dict(pos_scale=math.inf), dict(axes=1, dims=(66, 0, 0))]
BAD_ROWS = [dict(M=-1), dict(M=1 << 31), dict(H=-1), dict(Hk=-1), dict(H=0, Hk=0), dict(H=1025), dict(eps=-1e-6), dict(eps=math.nan),
            dict(eps=math.inf), dict(eps=0.0), dict(q_ld=255), dict(k_ld=127), dict(o_ld=255), dict(ko_ld=100), dict(q_ld=1 << 31),
            dict(q=None), dict(k=None), dict(o=None), dict(ko=None), dict(q=FAKE + 1), dict(ko=FAKE + 1), dict(gq=FAKE + 1)]


def _turn(lib, **kw):
    a = dict(q=FAKE, q_ld=256, k=FAKE, k_ld=128, M=9, H=4, Hk=2, d=64, gq=FAKE, gk=FAKE, eps=1e-6, rope=rope(), dtype=1, o=FAKE,
             o_ld=256, ko=FAKE, ko_ld=128)
    a.update(kw)
    return lib.avits_qk_norm_rope(*a.values(), None)


def test_qk_norm_rope(lib):
    for bad in BAD_ROWS:
        assert _turn(lib, **bad) == INVALID, bad
    for bad in BAD_ROPES:
        assert _turn(lib, rope=rope(**bad)) == INVALID, bad
    assert _turn(lib, d=96) == UNSUPPORTED and _turn(lib, dtype=2) == UNSUPPORTED
    assert _turn(lib, M=0, q=None, o=None, k=None, ko=None, rope=None) == 0


def _back(lib, **kw):
    a = dict(dqo=FAKE, dqo_ld=256, dko=FAKE, dko_ld=128, q=FAKE, q_ld=256, k=FAKE, k_ld=128, M=9, H=4, Hk=2, d=64, gq=FAKE,
             gk=FAKE, eps=1e-6, rope=rope(), dtype=1, o=FAKE, o_ld=256, ko=FAKE, ko_ld=128, dgq=FAKE, dgk=FAKE, ws=FAKE, wsb=BIG)
    a.update(kw)
    return lib.avits_qk_norm_rope_backward(*a.values(), None)


def test_qk_norm_rope_backward(lib):
    for bad in BAD_ROWS + [dict(dqo=None), dict(dko=None), dict(dqo=FAKE + 1), dict(dgq=FAKE + 2), dict(dqo_ld=200), dict(dko_ld=1 << 31),
                           dict(eps=0.0, gq=None, gk=None), dict(H=0), dict(ws=FAKE + 8)]:
        assert _back(lib, **bad) == INVALID, bad
    for bad in BAD_ROPES:
        assert _back(lib, rope=rope(**bad)) == INVALID, bad
    assert _back(lib, d=32) == UNSUPPORTED and _back(lib, dtype=-1) == UNSUPPORTED
    need = lib.avits_qk_norm_rope_backward_workspace_bytes(9, 4, 2, 64)
    assert need > 0 and _back(lib, ws=None) == WORKSPACE and _back(lib, wsb=need - 1) == WORKSPACE
    assert _back(lib, M=0, dgq=None, dgk=None) == 0
    sizes = [lib.avits_qk_norm_rope_backward_workspace_bytes(m, 4, 2, 64) for m in (0, 1, 9, 100, 2047, 2048, 2049, 5000, 10 ** 6)]
    assert sizes == sorted(sizes)          # a workspace suffices for fewer rows too
    for bad in ((-1, 4, 2, 64), (9, 0, 0, 64), (9, 1025, 2, 64), (9, 4, -1, 64), (9, 4, 2, 80), (1 << 31, 4, 2, 64)):
        assert lib.avits_qk_norm_rope_backward_workspace_bytes(*bad) == 0


def test_rope_frequencies(lib):
    f = avits.avits_rope_frequencies((8, 28, 0, 4)).numpy()
    want = np.concatenate([10000.0 ** (-2.0 * np.arange(n // 2) / max(n, 1)) for n in (8, 28, 0, 4)])
    assert np.allclose(f, want, rtol=1e-14)
    assert np.allclose(avits.avits_rope_frequencies((64,), theta=5e5, factor=4.0).numpy() * 4,
                       5e5 ** (-2.0 * np.arange(32) / 64), rtol=1e-14)
    # 4096 positions: pair m turns 4096 f / 2 pi times; between 1 and 32 turns the two are mixed.
    g = avits.avits_rope_frequencies((64,), factor=8.0, trained=4096, low=1.0, high=32.0).numpy()
    f = 10000.0 ** (-2.0 * np.arange(32) / 64)
    turns = 4096 * f / (2 * np.pi)
    keep = np.clip((turns - 1) / 31, 0, 1)
    assert np.allclose(g, f * keep + f / 8 * (1 - keep), rtol=1e-13) and keep[0] == 1 and keep[-1] == 0
    out = (ctypes.c_double * 64)()
    dims = (ctypes.c_int32 * 4)(8, 28, 28, 0)
    ok = dict(axes=3, dims=dims, theta=1e4, factor=1.0, trained=0, low=1.0, high=32.0, freq=out)
    for bad in (dict(axes=0), dict(axes=5), dict(dims=None), dict(freq=None), dict(theta=0.0), dict(theta=math.inf), dict(factor=0.0),
                dict(factor=math.nan), dict(trained=-1), dict(trained=8, low=-1.0), dict(trained=8, low=32.0),
                dict(trained=8, high=math.inf), dict(dims=(ctypes.c_int32 * 3)(8, 27, 28)), dict(dims=(ctypes.c_int32 * 3)(8, -2, 28))):
        assert lib.avits_rope_frequencies(*{**ok, **bad}.values()) == INVALID, bad


def _means(lib, **kw):
    a = dict(x=FAKE, ld=256, M=9, H=4, d=64, block=128, B=1, off=None, dtype=1, means=FAKE)
    a.update(kw)
    return lib.avits_block_means(*a.values(), None)


BAD_SEQS = [dict(B=0), dict(B=17), dict(B=2), dict(M=-1), dict(M=(1 << 31) - 4096)]


def test_block_means(lib):
    for bad in BAD_SEQS + [dict(block=100), dict(block=0), dict(H=0), dict(H=1025), dict(x=None), dict(means=None), dict(ld=255),
                           dict(ld=257), dict(x=FAKE + 2), dict(means=FAKE + 8), dict(off=arr(1, 9)), dict(off=arr(0, 10)),
                           dict(B=2, off=arr(0, 5, 4)), dict(ld=1 << 31)]:
        assert _means(lib, **bad) == INVALID, bad
    assert _means(lib, d=80) == UNSUPPORTED and _means(lib, dtype=2) == UNSUPPORTED
    assert _means(lib, M=0, x=None, means=None) == 0 and _means(lib, off=arr(0, 0), x=None) == 0


def _select(lib, **kw):
    a = dict(qm=FAKE, km=FAKE, M=300, N=900, B=1, qo=None, ko=None, H=4, Hk=2, d=64, q_lead=0, k_lead=0, keep=3, mask=FAKE, words=1)
    a.update(kw)
    return lib.avits_block_select(*a.values(), None)


def test_block_select(lib):
    for bad in BAD_SEQS + [dict(N=-1), dict(qo=arr(0, 301)), dict(ko=arr(1, 900)), dict(Hk=0), dict(Hk=3), dict(H=0), dict(H=2048, Hk=1),
                           dict(H=1, Hk=2), dict(q_lead=-1), dict(k_lead=-1), dict(keep=-1), dict(words=0), dict(words=-1),
                           dict(N=64 * 64 + 1), dict(qm=None), dict(km=None), dict(mask=None), dict(qm=FAKE + 8), dict(mask=FAKE + 4)]:
        assert _select(lib, **bad) == INVALID, bad
    assert _select(lib, d=32) == UNSUPPORTED
    assert _select(lib, N=16385 * 64, words=300) == UNSUPPORTED
    assert _select(lib, M=0, qm=None, mask=None) == 0


def rows(p=FAKE, ld=256):
    return ctypes.byref(B._Rows(p, ld))


def _attend(lib, **kw):
    a = dict(q=rows(), k=rows(ld=128), v=rows(ld=128), M=300, N=900, B=1, qo=None, ko=None, H=4, Hk=2, d=64, mask=FAKE, words=1, scale=0.1,
             dtype=1, o=rows(), lse=None, ws=FAKE, wsb=BIG)
    a.update(kw)
    return lib.avits_sparse_attention(*a.values(), None)


BAD_ATTN = BAD_SEQS + [dict(N=-1), dict(qo=arr(0, 301)), dict(ko=arr(1, 900)), dict(Hk=0), dict(Hk=3), dict(H=0), dict(H=2048, Hk=1),
                       dict(words=0), dict(words=-1), dict(N=64 * 64 + 1), dict(mask=FAKE + 4), dict(scale=0.0), dict(scale=-1.0),
                       dict(scale=math.nan), dict(scale=math.inf), dict(q=None), dict(q=rows(None)), dict(q=rows(ld=255)), dict(q=rows(ld=260)),
                       dict(q=rows(FAKE + 8)), dict(q=rows(ld=1 << 24)), dict(k=None), dict(v=rows(None)), dict(k=rows(ld=120)),
                       dict(v=rows(ld=132)), dict(o=None), dict(o=rows(None)), dict(o=rows(ld=128))]


def test_sparse_attention(lib):
    for bad in BAD_ATTN:
        assert _attend(lib, **bad) == INVALID, bad
    assert _attend(lib, d=96) == UNSUPPORTED and _attend(lib, dtype=2) == UNSUPPORTED
    assert _attend(lib, M=0, q=rows(None), o=rows(None)) == 0


def _attend_back(lib, **kw):
    a = dict(dout=rows(), q=rows(), k=rows(ld=128), v=rows(ld=128), o=rows(), lse=FAKE, M=300, N=900, B=1, qo=None, ko=None, H=4, Hk=2, d=64,
             mask=FAKE, words=1, scale=0.1, dtype=1, dq=rows(), dk=rows(ld=128), dv=rows(ld=128), ws=FAKE, wsb=BIG)
    a.update(kw)
    return lib.avits_sparse_attention_backward(*a.values(), None)


def test_sparse_attention_backward(lib):
    for bad in BAD_ATTN + [dict(dout=None), dict(dq=rows(None)), dict(dk=rows(ld=100)), dict(dv=None), dict(lse=None), dict(ws=FAKE + 8)]:
        assert _attend_back(lib, **bad) == INVALID, bad
    assert _attend_back(lib, d=96) == UNSUPPORTED and _attend_back(lib, dtype=2) == UNSUPPORTED
    need = lib.avits_sparse_attention_backward_workspace_bytes(300, 900, 1, 4, 2, 64, 1)
    assert need > 0 and _attend_back(lib, ws=None) == WORKSPACE and _attend_back(lib, wsb=need - 1) == WORKSPACE
    assert _attend_back(lib, M=0, N=0) == 0


def test_binding_refuses_before_the_library():
    import torch
    q, k = torch.zeros(5, 4, 64), torch.zeros(5, 2, 64)
    with pytest.raises(ValueError, match="neither"):
        avits.avits_qk_norm_rope(None, None, None, None)
    with pytest.raises(ValueError, match="both pos and freq"):
        avits.avits_qk_norm_rope(q, k, q, k, freq=torch.zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError, match="sum to 64"):
        avits.avits_qk_norm_rope(q, k, q, k, pos=torch.zeros(5, 2, dtype=torch.int32), freq=torch.zeros(32, dtype=torch.float64), dims=(8, 28))
    with pytest.raises(ValueError, match="do not reach"):
        avits.avits_sparse_attention(q, k, k, q, mask=torch.zeros(4, 1, 0, dtype=torch.int64))
    with pytest.raises(ValueError, match="sequences"):
        avits.avits_sparse_attention(q, k, k, q, q_off=[0, 2, 5], k_off=[0, 5])
    with pytest.raises(ValueError, match="match the offsets"):
        avits.avits_block_select(torch.zeros(2, 4, 64), k, 1, torch.zeros(4, 2, 1), q_off=[0, 128], k_off=[0, 320])
    if not torch.cuda.is_available():
        with pytest.raises(avits.AvitsError):
            avits.avits_qk_norm_rope(q, k, q, k)
        with pytest.raises(avits.AvitsError):
            avits.avits_sparse_attention(q, k, k, q)
        with pytest.raises(avits.AvitsError):
            avits.avits_qk_norm_rope(q.to(torch.float16), k, q, k)


def test_scales_and_workspaces(lib):
    """Scales whose logits or their inverses leave fp32 are refused; a workspace does for fewer rows, sequences and keys."""
    for bad in (2.0 ** -65, 2.0 ** 65, 1e-45):
        assert _attend(lib, scale=bad) == INVALID and _attend_back(lib, scale=bad) == INVALID, bad
    forward, backward = lib.avits_sparse_attention_workspace_bytes, lib.avits_sparse_attention_backward_workspace_bytes
    for H, Hk in ((1, 1), (4, 2), (16, 16), (1024, 1)):
        sizes = [(forward(m, m, b, H, 128, 1), backward(m, m, b, H, Hk, 128, 1))
                 for m, b in ((0, 1), (1, 1), (64, 1), (65, 2), (700, 2), (1100, 2), (2047, 3), (4608, 3), (5000, 16), (16896, 16), (200000, 16))]
        assert sizes == sorted(sizes) and [s[1] for s in sizes] == sorted(s[1] for s in sizes)
    assert forward(4608, 4608, 1, 16, 128, 0) == 0 and forward(-1, 5, 1, 4, 64, 1) == 0 and backward(5, 5, 17, 4, 2, 64, 1) == 0
    # Too small by a byte wherever one is needed: one row of long lists, few units, a plan.
    for M, N, H, Hk in ((1, 9000, 4, 4), (300, 2900, 4, 2), (1500, 1500, 8, 8)):
        a = dict(q=rows(ld=H * 64), k=rows(ld=H * 64), v=rows(ld=H * 64), o=rows(ld=H * 64), M=M, N=N, H=H, Hk=Hk, words=3)
        assert _attend(lib, **a, ws=None) == WORKSPACE and _attend(lib, **a, wsb=64) == WORKSPACE
        assert _attend(lib, **a, ws=FAKE + 8) == INVALID

"""Refusals of the low-bit and training entry points: every call below fails
on the host, before any device memory is touched (or has nothing to do)."""
import ctypes

import pytest

import paper_2608_17995_amd as avits

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
FAKE = 0x1000  # never dereferenced
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return avits.load()


def arr(*v):
    return (ctypes.c_int64 * len(v))(*v)


def _norm(lib, **kw):
    a = dict(x=FAKE, M=8, D=16, B=1, off=None, sh=FAKE, sc=FAKE, stride=0, eps=1e-6, dtype=1, h=FAKE, mean=FAKE, rstd=FAKE)
    a.update(kw)
    return lib.avits_layer_norm(a["x"], a["M"], a["D"], a["B"], a["off"], a["sh"], a["sc"], a["stride"], a["eps"],
                                a["dtype"], a["h"], a["mean"], a["rstd"], None)


def test_layer_norm(lib):
    for bad in (dict(M=-1), dict(M=1 << 26), dict(D=0), dict(D=65537), dict(B=0), dict(B=17, off=arr(*range(18))), dict(B=2),
                dict(off=arr(1, 8)), dict(off=arr(0, 7)), dict(B=2, off=arr(0, 9, 8)), dict(stride=-1), dict(eps=0.0),
                dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(h=None),
                dict(x=FAKE + 1), dict(sc=FAKE + 1), dict(mean=FAKE + 2)):
        assert _norm(lib, **bad) == INVALID, bad
    assert _norm(lib, dtype=2) == UNSUPPORTED
    assert _norm(lib, M=0, x=None, h=None) == 0
    assert b"eps" in (_norm(lib, eps=0.0), lib.avits_last_error())[1]


def _back(lib, **kw):
    a = dict(dh=FAKE, x=FAKE, q=None, s=None, mean=FAKE, rstd=FAKE, M=8, D=16, B=1, off=None, sc=FAKE, stride=0, dres=None,
             dtype=1, dx=FAKE, dsc=FAKE, dsh=FAKE, ws=FAKE, wsb=BIG)
    a.update(kw)
    return lib.avits_layer_norm_backward(a["dh"], a["x"], a["q"], a["s"], a["mean"], a["rstd"], a["M"], a["D"], a["B"],
                                         a["off"], a["sc"], a["stride"], a["dres"], a["dtype"], a["dx"], a["dsc"], a["dsh"],
                                         a["ws"], a["wsb"], None)


def test_layer_norm_backward(lib):
    for bad in (dict(x=None), dict(q=FAKE, s=FAKE), dict(x=None, q=FAKE), dict(x=None, s=FAKE), dict(s=FAKE), dict(dh=None),
                dict(mean=None), dict(rstd=None), dict(dx=None), dict(M=-1), dict(D=0), dict(B=2), dict(stride=-2),
                dict(dres=FAKE + 1), dict(dsc=FAKE + 2)):
        assert _back(lib, **bad) == INVALID, bad
    assert _back(lib, dtype=5) == UNSUPPORTED
    need = lib.avits_layer_norm_backward_workspace_bytes(8, 16, 1)
    assert need > 0
    assert _back(lib, ws=None) == WORKSPACE and _back(lib, wsb=need - 1) == WORKSPACE
    assert _back(lib, M=0, dsc=None, dsh=None) == 0
    for bad in ((-1, 16, 1), (8, 0, 1), (8, 16, 0), (8, 16, 17), (1 << 26, 16, 1)):
        assert lib.avits_layer_norm_backward_workspace_bytes(*bad) == 0


def test_activations_in_8_bits(lib):
    for f, order in ((lib.avits_ckpt8_pack, "pack"), (lib.avits_ckpt8_unpack, "unpack")):
        call = (lambda x, M, D, dt, q, s: f(x, M, D, dt, q, s, None)) if order == "pack" else \
               (lambda x, M, D, dt, q, s: f(q, s, M, D, dt, x, None))
        for bad in ((None, 4, 8, 1, FAKE, FAKE), (FAKE, 4, 8, 1, None, FAKE), (FAKE, 4, 8, 1, FAKE, None),
                    (FAKE, -1, 8, 1, FAKE, FAKE), (FAKE, 1 << 31, 8, 1, FAKE, FAKE), (FAKE, 4, 0, 1, FAKE, FAKE),
                    (FAKE, 4, 1 << 24, 1, FAKE, FAKE), (FAKE + 1, 4, 8, 1, FAKE, FAKE), (FAKE + 2, 4, 8, 0, FAKE, FAKE)):
            assert call(*bad) == INVALID, (order, bad)
        assert call(FAKE, 4, 8, 3, FAKE, FAKE) == UNSUPPORTED
        assert call(None, 0, 8, 1, None, None) == 0
    g = lib.avits_gelu_backward
    for bad in ((FAKE, None, None, None, 4, 8, 1, FAKE), (FAKE, FAKE, FAKE, FAKE, 4, 8, 1, FAKE),
                (FAKE, None, FAKE, None, 4, 8, 1, FAKE), (None, FAKE, None, None, 4, 8, 1, FAKE),
                (FAKE, FAKE, None, None, 4, 8, 1, None), (FAKE, FAKE, None, None, -4, 8, 1, FAKE),
                (FAKE, FAKE + 1, None, None, 4, 8, 1, FAKE)):
        assert g(*bad, None) == INVALID, bad
    assert g(FAKE, FAKE, None, None, 4, 8, 9, FAKE, None) == UNSUPPORTED
    assert g(None, FAKE, None, None, 0, 8, 1, None, None) == 0


def test_quantisation(lib):
    def q(x=FAKE, M=4, K=64, act=0, dt=1, q=FAKE, s=FAKE):
        return lib.avits_mxfp4_quantize(x, M, K, act, dt, q, s, None)

    def d(x=FAKE, M=4, K=64, dt=1, q=FAKE, s=FAKE):
        return lib.avits_mxfp4_dequantize(q, s, M, K, dt, x, None)

    for f in (q, d):
        for bad in (dict(x=None), dict(q=None), dict(s=None), dict(M=-1), dict(M=1 << 28), dict(K=0), dict(K=48), dict(K=33),
                    dict(K=1 << 24), dict(M=1 << 27, K=1 << 10), dict(x=FAKE + 8), dict(q=FAKE + 4), dict(s=FAKE + 2)):
            assert f(**bad) == INVALID, bad
        assert f(dt=2) == UNSUPPORTED
        assert f(M=0, x=None, q=None, s=None) == 0
    assert q(act=2) == INVALID
    size = lib.avits_mxfp4_scale_bytes
    assert size(1, 32) == 16 and size(8, 64) == 16 and size(9, 96) == 64 and size(0, 64) == 0
    assert size(-1, 64) == 0 and size(4, 40) == 0
    assert avits.avits_mxfp4_scale_shape(9, 96) == (2, 16, 2)


def _linear(lib, **kw):
    a = dict(xq=FAKE, xs=FAKE, M=4, K=64, wq=FAKE, ws=FAKE, b=FAKE, N=8, B=1, off=None, gate=None, stride=0, resid=None,
             dtype=1, out=FAKE, work=FAKE, wb=BIG)
    a.update(kw)
    return lib.avits_mxfp4_linear(a["xq"], a["xs"], a["M"], a["K"], a["wq"], a["ws"], a["b"], a["N"], a["B"], a["off"],
                                  a["gate"], a["stride"], a["resid"], a["dtype"], a["out"], a["work"], a["wb"], None)


def _lback(lib, **kw):
    a = dict(dy=FAKE, M=4, N=8, wq=FAKE, ws=FAKE, K=64, dtype=1, dx=FAKE, work=FAKE, wb=BIG)
    a.update(kw)
    return lib.avits_mxfp4_linear_backward(a["dy"], a["M"], a["N"], a["wq"], a["ws"], a["K"], a["dtype"], a["dx"],
                                           a["work"], a["wb"], None)


def test_products(lib):
    sizes = (dict(M=-1), dict(M=1 << 28), dict(N=0), dict(N=1 << 21), dict(K=0), dict(K=48), dict(K=1 << 21),
             dict(M=1 << 27, K=1 << 10), dict(wq=None), dict(ws=None), dict(wq=FAKE + 8), dict(ws=FAKE + 8))
    for bad in sizes + (dict(xq=None), dict(xs=None), dict(out=None), dict(gate=FAKE), dict(resid=FAKE), dict(B=2),
                        dict(B=0), dict(off=arr(0, 3)), dict(stride=-1), dict(out=FAKE + 2), dict(b=FAKE + 1),
                        dict(gate=FAKE, resid=FAKE + 8)):
        assert _linear(lib, **bad) == INVALID, bad
    for bad in sizes + (dict(dy=None), dict(dx=None), dict(dy=FAKE + 2), dict(dx=FAKE + 8), dict(work=FAKE + 8)):
        assert _lback(lib, **bad) == INVALID, bad
    assert _linear(lib, dtype=2) == UNSUPPORTED and _lback(lib, dtype=2) == UNSUPPORTED
    assert _linear(lib, M=0, xq=None, out=None) == 0 and _lback(lib, M=0, dy=None, dx=None) == 0
    need = lib.avits_mxfp4_linear_backward_workspace_bytes(4, 8, 64, 1)
    assert need >= 64 * 8 * 2
    assert _lback(lib, work=None) == WORKSPACE and _lback(lib, wb=need - 1) == WORKSPACE
    assert lib.avits_mxfp4_linear_backward_workspace_bytes(4, 8, 40, 1) == 0
    # A product split along its contraction needs its parts' room; the query covers every smaller M.
    need = lib.avits_mxfp4_linear_workspace_bytes(512, 256, 8192)
    assert need >= lib.avits_mxfp4_linear_workspace_bytes(300, 256, 8192) > 0
    assert _linear(lib, M=1741, N=2048, K=8192, work=None) == WORKSPACE
    assert _linear(lib, M=1741, N=2048, K=8192, wb=1024) == WORKSPACE
    assert _linear(lib, M=1741, N=2048, K=8192, work=FAKE + 8) == INVALID
    assert lib.avits_mxfp4_linear_workspace_bytes(512, 256, 256) == 0 and lib.avits_mxfp4_linear_workspace_bytes(0, 8, 64) == 0


def test_the_binding_refuses_shapes_and_types():
    torch = pytest.importorskip("torch")
    z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t)  # noqa: E731  (CPU tensors: nothing can be launched)
    with pytest.raises((ValueError, avits.AvitsError)):
        avits.avits_layer_norm(z(4, 8), None, None, z(4, 9))
    with pytest.raises((ValueError, avits.AvitsError)):
        avits.avits_layer_norm(z(4, 8), None, None, z(4, 8))          # not on the GPU
    with pytest.raises((ValueError, avits.AvitsError)):
        avits.avits_layer_norm(z(4, 8), z(8), None, z(4, 8))
    with pytest.raises((ValueError, avits.AvitsError)):
        avits.avits_layer_norm(z(4, 8), None, None, z(4, 8), off=[4])
    with pytest.raises((ValueError, avits.AvitsError)):
        avits.avits_layer_norm_backward(z(4, 8), z(4), z(3), None, z(4, 8), x=z(4, 8))
    with pytest.raises((ValueError, avits.AvitsError)):
        avits.avits_ckpt8_pack(z(4, 40), z(4, 40, t=torch.uint8), z(4, 1, t=torch.uint8))
    with pytest.raises((ValueError, avits.AvitsError)):
        avits.avits_gelu_backward(z(4, 8), z(4, 8), m=z(4, 7))
    u = torch.uint8
    with pytest.raises((ValueError, avits.AvitsError)):
        avits.avits_mxfp4_quantize(z(4, 64), z(4, 32, t=u), z(1, 4, 2, t=u))
    with pytest.raises((ValueError, avits.AvitsError)):
        avits.avits_mxfp4_linear(z(4, 32, t=u), z(1, 8, 2, t=u), z(8, 48, t=u), z(2, 8, 2, t=u), None, z(4, 8))
    with pytest.raises((ValueError, avits.AvitsError)):
        avits.avits_mxfp4_linear_backward(z(4, 9), z(8, 32, t=u), z(1, 8, 2, t=u), z(4, 64))


def test_the_largest_sizes(lib):
    """What a launch's 2^32 work-items cannot hold is refused."""
    assert _norm(lib, M=1 << 25) == INVALID and _back(lib, M=1 << 25) == INVALID
    assert lib.avits_layer_norm_backward_workspace_bytes((1 << 25) - 1, 1, 1) > 0
    assert lib.avits_mxfp4_quantize(FAKE, 1 << 27, 32, 0, 1, FAKE, FAKE, None) == INVALID
    assert lib.avits_mxfp4_dequantize(FAKE, FAKE, 1 << 27, 32, 1, FAKE, None) == INVALID
    assert lib.avits_mxfp4_scale_bytes(1 << 27, 32) == 0 and lib.avits_mxfp4_scale_bytes((1 << 27) - 1, 32) == 1 << 28
    assert _linear(lib, M=1 << 27, K=32) == INVALID and _lback(lib, M=1 << 27, K=32) == INVALID


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("N,K", [(8, 32), (9, 64), (256, 1024), (2048, 8192), (4100, 1056)])
def test_workspaces_cover_fewer_rows(lib, N, K, dtype):
    sizes = [1, 2, 15, 16, 17, 64, 65, 200, 256, 257, 300, 512, 777, 1024, 1741, 4096, 16896, 70000]
    for query in (lambda M: lib.avits_mxfp4_linear_workspace_bytes(M, N, K),
                  lambda M: lib.avits_mxfp4_linear_backward_workspace_bytes(M, N, K, dtype),
                  lambda M: lib.avits_layer_norm_backward_workspace_bytes(M, K, 4)):
        need = [query(M) for M in sizes]
        assert need == sorted(need)


def test_tensors_elsewhere_are_refused():
    """Everything is on the current device, or nothing is launched: here there is none."""
    torch = pytest.importorskip("torch")
    z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t)  # noqa: E731
    u, meta = torch.uint8, torch.zeros(4, 64, device="meta")
    for x in (z(4, 64), meta):
        with pytest.raises(avits.AvitsError):
            avits.avits_layer_norm(x, None, None, x)
        with pytest.raises(avits.AvitsError):
            avits.avits_layer_norm_backward(x, z(4), z(4), None, x, x=x)
        with pytest.raises(avits.AvitsError):
            avits.avits_ckpt8_pack(x, z(4, 64, t=u), z(4, 2, t=u))
        with pytest.raises(avits.AvitsError):
            avits.avits_ckpt8_unpack(z(4, 64, t=u), z(4, 2, t=u), x)
        with pytest.raises(avits.AvitsError):
            avits.avits_gelu_backward(x, x, m=x)
        with pytest.raises(avits.AvitsError):
            avits.avits_mxfp4_quantize(x, z(4, 32, t=u), z(1, 8, 2, t=u))
        with pytest.raises(avits.AvitsError):
            avits.avits_mxfp4_dequantize(z(4, 32, t=u), z(1, 8, 2, t=u), x)
        with pytest.raises(avits.AvitsError):
            avits.avits_mxfp4_linear(z(8, 16, t=u), z(1, 8, 2, t=u), z(64, 16, t=u), z(1, 64, 2, t=u), None, x[:, :].new_zeros(8, 64))
        with pytest.raises(avits.AvitsError):
            avits.avits_mxfp4_linear_backward(x, z(64, 16, t=u), z(1, 64, 2, t=u), x[:, :32], workspace=z(64, t=u))

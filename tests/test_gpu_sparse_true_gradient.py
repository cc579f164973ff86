"""bf16: the gradients from the forward's own o and lse against the exact gradient of the inputs, for which o and lse are
taken in 64 bits.  Besides the backward pass's own roundings delta = dout . o carries those of o."""
import pytest

from _sparse import backward, forward, make

pytestmark = pytest.mark.gpu

U, LOW = 2.0 ** -24, 2.0 ** -8


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("M", [3, 110, 700])
@pytest.mark.parametrize("shared", [0, 8])
def test_exact_gradient(gpu, shared, M, d):
    import torch
    H, Hk = 4, 2
    s = make(H, Hk, d, (0, M), (0, M), "bf16", seed=81, extra=0, packed=False)
    # `shared`: how much all keys of a head have in common, against a spread of 1.
    s["k"] = (s["k"].float() + shared * torch.randn(1, Hk, d, generator=torch.Generator().manual_seed(82)).cuda()).to(torch.bfloat16)
    if shared:
        s["q"].mul_(0.25)
    forward(gpu, s, mask=None)
    backward(gpu, s, mask=None)
    q, k, v, do = (s[n].double() for n in ("q", "k", "v", "do"))
    scale = s["scale"]
    want = [torch.zeros_like(t) for t in (q, k, v)]
    tol = [torch.zeros_like(t) for t in (q, k, v)]
    for h in range(H):
        j = h // (H // Hk)
        x = q[:, h] @ k[:, j].T.contiguous() * scale
        lse = torch.logsumexp(x, 1, keepdim=True)
        p = torch.exp(x - lse)
        o = p @ v[:, j]
        g = do[:, h]
        ds = p * (g @ v[:, j].T.contiguous() - (g * o).sum(1, keepdim=True))
        want[0][:, h], want[1][:, j], want[2][:, j] = scale * ds @ k[:, j], want[1][:, j] + scale * ds.T @ q[:, h], want[2][:, j] + p.T @ g
        # A logit: d products in fp32, scaled; its exponential.  lse: the same, its sum's M / 4 + 40 roundings and its own.
        es = U * ((d + 2) * (q[:, h].abs() @ k[:, j].T.abs().contiguous()) * scale + 4 * x.abs() + 6)
        el = es.max(1, keepdim=True).values + U * (M / 4 + 40 + 4 * lse.abs() + 4 * x.abs().max(1, keepdim=True).values)
        ep = p * (es + el + 4 * U)
        # o: the probabilities' rounding to bf16 and errors, then its own rounding; so delta.
        size = p @ v[:, j].abs()
        eo = (LOW + 2 * es.max(1, keepdim=True).values + U * (M / 4 + 40)) * size
        eo = eo + LOW * (o.abs() + eo)
        terms = g.abs() @ v[:, j].T.abs().contiguous() + (g.abs() * (o.abs() + eo)).sum(1, keepdim=True)
        eds = ds.abs() * (es + el + 4 * U) + p * ((g.abs() * eo).sum(1, keepdim=True) + U * (d + 4) * terms)
        chain = U * ((H // Hk) * M / 4 + 20)
        # ds for dq in two parts of 8 bits, 2^-16; ds for dk and p for dv in one.
        tol[0][:, h] = scale * (eds + (2.0 ** -16 + chain) * (ds.abs() + eds)) @ k[:, j].abs()
        tol[1][:, j] += scale * (eds + (LOW + chain) * (ds.abs() + eds)).T @ q[:, h].abs()
        tol[2][:, j] += (ep + (LOW + chain) * (p + ep)).T @ g.abs()
    for n, w, t in zip(("dq", "dk", "dv"), want, tol):
        err = (s[n].double() - w).abs()
        bound = t + LOW * (w.abs() + t)
        assert (err <= bound).all(), (n, float((err / bound).max()))

"""Inputs of the sparse attention tests, and bounds from the arithmetic."""
import numpy as np
import torch

import oracle
from _bounds import assert_within
from _gpu import TORCH_DT, rel_l2

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}


def np64(t):
    return t.double().cpu().numpy()


def make(H, Hk, d, q_off, k_off, dtype, seed=0, density=0.4, extra=3, packed=True):
    """Rows (a few behind the last sequence), outputs filled with 5, a random mask with an empty row of blocks."""
    g = torch.Generator().manual_seed(seed)
    dt = TORCH_DT[dtype]
    M, N = q_off[-1] + extra, k_off[-1] + extra
    n = lambda rows, *heads: torch.randn(rows, sum(heads), d, generator=g).to(dt).cuda().split(list(heads), 1)  # noqa: E731
    s = dict(dtype=dtype, q_off=q_off, k_off=k_off, scale=d ** -0.5)
    if packed and M == N:
        s["q"], s["k"], s["v"] = n(M, H, Hk, Hk)
    else:
        s["q"], (s["k"], s["v"]) = n(M, H)[0], n(N, Hk, Hk)
    s["do"] = n(M, H, 1)[0]
    qs, ks = oracle.cut(q_off, 128), oracle.cut(k_off, 64)
    nk = [sum(b == i for b, _, _ in ks) for i in range(len(k_off) - 1)]
    on = np.random.default_rng(seed).random((H, len(qs), max(nk))) < density
    on[H // 2, len(qs) // 2:len(qs) // 2 + 1] = False
    s["on"] = on
    s["mask"] = torch.from_numpy(oracle.words(on, -(-max(nk) // 64) + 1).copy()).cuda() if max(nk) else \
        torch.zeros(H, len(qs), 1, dtype=torch.int64, device="cuda")
    s["mask"][:, :, -1] |= -(1 << 63)      # bits past the last key block count for nothing
    five = lambda *shape, dt=dt: torch.full(shape, 5.0, dtype=dt, device="cuda")  # noqa: E731
    s.update(o=five(M, H, d), lse=five(H, M, dt=torch.float32))
    s["dq"], s["dk"], s["dv"] = five(M, H + 2, d)[:, :H], five(N, Hk, d), five(N, Hk + 1, d)[:, :Hk]
    return s


def forward(gpu, s, **kw):
    a = dict(mask=s["mask"], lse=s["lse"], q_off=s["q_off"], k_off=s["k_off"])
    gpu.avits_sparse_attention(s["q"], s["k"], s["v"], s["o"], **{**a, **kw})


def backward(gpu, s, **kw):
    a = dict(mask=s["mask"], q_off=s["q_off"], k_off=s["k_off"])
    gpu.avits_sparse_attention_backward(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["dq"], s["dk"], s["dv"], **{**a, **kw})


def check_forward(s, on="mask"):
    q, k, v = np64(s["q"]), np64(s["k"]), np64(s["v"])
    M, H, d = q.shape
    g, m = H // k.shape[1], s["q_off"][-1]
    ok = oracle.allowed(s["on"] if isinstance(on, str) else on, s["q_off"], s["k_off"], M, len(k))
    o, lse = oracle.sparse_attention(q, k, v, ok, s["scale"])
    half = HALF[s["dtype"]]
    got, got_lse = np64(s["o"]), s["lse"].double().cpu().numpy()
    assert (got[m:] == 5).all() and (got_lse[:, m:] == 5).all()
    for h in range(H):
        w = ok[h % len(ok)][:m]
        # A logit: d products summed in fp32, scaled; its exponential 3 roundings and the logit's size twice.
        es = U * ((d + 2) * (np.abs(q[:m, h]) @ np.abs(k[:, h // g]).T) * s["scale"])
        es = np.where(w, es, 0).max(1, initial=0) + 4 * U
        some = w.any(1)
        assert (got[:m, h][~some] == 0).all() and (got_lse[h, :m][~some] == -np.inf).all()
        x = np.where(w, q[:m, h] @ k[:, h // g].T * s["scale"], -np.inf)[some]
        p = np.exp(x - lse[h, :m][some][:, None])
        size = p @ np.abs(v[:, h // g])
        n = w.sum(1)[some]
        err = (2 * es[some] + U * (n / 4 + 40))[:, None] * size + (0 if s["dtype"] == "f32" else 2.0 ** -8) * size
        want = o[:m, h][some]
        assert_within(got[:m, h][some], want, err + half * (np.abs(want) + err), f"o, head {h}")
        top = np.abs(x[np.isfinite(x)]).max(initial=0)
        assert_within(got_lse[h, :m][some], lse[h, :m][some], es[some] + U * (n / 4 + 40 + 4 * np.abs(lse[h, :m][some]) + 4 * top), "lse")
    if s["dtype"] == "bf16" and np.any(o):
        assert rel_l2(got[:m], o[:m]) <= 2.0 ** -8    # two roundings of a third of a half step each, rms


def check_backward(s, on="mask"):
    """From the o and lse that the tensors hold."""
    q, k, v, do = np64(s["q"]), np64(s["k"]), np64(s["v"]), np64(s["do"])
    M, H, d = q.shape
    m, n = s["q_off"][-1], s["k_off"][-1]
    g = H // k.shape[1]
    scale, half = s["scale"], HALF[s["dtype"]]
    low = 0 if s["dtype"] == "f32" else 2.0 ** -8
    ok = oracle.allowed(s["on"] if isinstance(on, str) else on, s["q_off"], s["k_off"], M, len(k))
    o, lse = np64(s["o"]), s["lse"].double().cpu().numpy()
    want = oracle.sparse_attention_backward(do, q, k, v, o, np.where(np.isinf(lse), 0, lse), ok, scale)
    tol = [np.zeros_like(t) for t in want]
    for h in range(H):
        j, w = h // g, ok[h % len(ok)]
        x = q[:, h] @ k[:, j].T * scale
        ref = np.where(np.isinf(lse[h]), 0, lse[h])[:, None]
        p = np.where(w, np.exp(np.where(w, x - ref, 0)), 0)
        dp, delta = do[:, h] @ v[:, j].T, (do[:, h] * o[:, h]).sum(1)[:, None]
        es = U * ((d + 2) * (np.abs(q[:, h]) @ np.abs(k[:, j]).T) * scale + 4 * np.abs(x) + 4 * np.abs(ref) + 6)
        size = np.abs(do[:, h]) @ np.abs(v[:, j]).T + (np.abs(do[:, h]) * np.abs(o[:, h])).sum(1)[:, None]
        ds = p * np.abs(dp - delta)
        eds = ds * (es + 4 * U + low) + p * U * (d + 4) * size
        ep = p * (es + 4 * U + low)
        chain = U * (max(w.sum(1).max(initial=0), w.sum(0).max(initial=0) * g) / 4 + 20)
        tol[0][:, h] += scale * (eds + chain * ds) @ np.abs(k[:, j])
        tol[1][:, j] += scale * (eds + chain * ds).T @ np.abs(q[:, h])
        tol[2][:, j] += (ep + chain * p).T @ np.abs(do[:, h])
    for name, t, ref, rows in (("dq", tol[0], want[0], m), ("dk", tol[1], want[1], n), ("dv", tol[2], want[2], n)):
        got = np64(s[name])
        assert (got[rows:] == 5).all(), f"{name}: rows behind the last sequence"
        assert_within(got[:rows], ref[:rows], t[:rows] + half * (np.abs(ref[:rows]) + t[:rows]), name)
        if s["dtype"] == "bf16" and np.any(ref):
            # Besides the result's own rounding that of p or ds, and of o in delta, as large as a term can be.
            assert rel_l2(got[:rows], ref[:rows]) <= 2.0 ** -7, name

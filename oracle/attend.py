"""The attention half of a block by its parts, fp64: norm and rotation of queries
and keys, the choice of key blocks, attention over chosen blocks, and the gradients.

Test infrastructure: used only by tests.  Every function states the definition,
with no regard to speed.
"""
from __future__ import annotations

import numpy as np

QB, KB = 128, 64


def rope_turns(pos, freq, dims, pos_scale):
    """Angles [M, rot / 2] of positions [M, axes]."""
    axis = np.repeat(np.arange(len(dims)), [n // 2 for n in dims])
    return np.asarray(pos, np.float64)[:, axis] * pos_scale * np.asarray(freq, np.float64)


def pair_index(rot, halves):
    """Elements (first, second) of each pair of the rotated part."""
    m = np.arange(rot // 2)
    return (m, m + rot // 2) if halves else (2 * m, 2 * m + 1)


def turn(y, angles, halves):
    """y [M, H, d] with its leading pairs turned."""
    out = np.array(y, np.float64)
    a, b = pair_index(2 * angles.shape[1], halves)
    c, s = np.cos(angles)[:, None], np.sin(angles)[:, None]
    out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., a] * s + y[..., b] * c
    return out


def norm_turn(x, g, eps, angles, halves):
    """RMS norm (eps 0: none), gain and rotation of x [M, H, d]."""
    x = np.asarray(x, np.float64)
    if eps > 0:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if g is not None:
        x = x * np.asarray(g, np.float64)
    return x if angles is None else turn(x, angles, halves)


def norm_turn_backward(dy, x, g, eps, angles, halves):
    """(dx, dg) of norm_turn."""
    e = np.asarray(dy, np.float64)
    if angles is not None:
        e = turn(e, -angles, halves)
    if eps <= 0:
        return e, None
    x = np.asarray(x, np.float64)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    dg = (e * n).sum((0, 1))
    if g is not None:
        e = e * np.asarray(g, np.float64)
    return r * (e - n * (e * n).mean(-1, keepdims=True)), dg


def cut(off, size):
    """Each block's (sequence, first row, end row)."""
    return [(b, i, min(i + size, hi)) for b, (lo, hi) in enumerate(zip(off, off[1:])) for i in range(lo, hi, size)]


def block_means(x, off, size):
    x = np.asarray(x, np.float64)
    return np.array([x[lo:hi].sum(0) / (hi - lo) for _, lo, hi in cut(off, size)]).reshape(-1, *x.shape[1:])


def block_select(q_means, k_means, keep, q_off, k_off, q_lead=0, k_lead=0):
    """Truth values [H, query blocks, most key blocks of a sequence]."""
    H, Hk = q_means.shape[1], k_means.shape[1]
    qs, ks = cut(q_off, QB), cut(k_off, KB)
    at = [[j for j, (b, _, _) in enumerate(ks) if b == s] for s in range(len(k_off) - 1)]
    on = np.zeros((H, len(qs), max(len(a) for a in at)), bool)
    for h in range(H):
        for i, (b, lo, _) in enumerate(qs):
            n = len(at[b])
            local = np.arange(n)
            lead = local * KB < k_lead
            if lo - q_off[b] < q_lead:
                on[h, i, :n] = True
                continue
            s = k_means[at[b], h // (H // Hk)] @ q_means[i, h]
            nan = np.isnan(s)
            order = np.lexsort((local, -np.where(nan, 0, s), nan, lead))
            on[h, i, order[:min(keep, n - lead.sum())]] = True
            on[h, i, :n] |= lead
    return on


def words(on, n_words=None):
    """The mask's int64 words of truth values [..., key blocks]."""
    n = n_words or -(-on.shape[-1] // 64)
    bits = np.zeros((*on.shape[:-1], 64 * n), np.uint64)
    bits[..., :on.shape[-1]] = on
    return (bits.reshape(*on.shape[:-1], n, 64) << np.arange(64, dtype=np.uint64)).sum(-1, dtype=np.uint64).view(np.int64)


def allowed(on, q_off, k_off, M, N):
    """Truth values [H, M, N]: which keys each query attends to (None: all of its sequence)."""
    qs, ks = cut(q_off, QB), cut(k_off, KB)
    H = 1 if on is None else len(on)
    out = np.zeros((H, M, N), bool)
    for i, (b, lo, hi) in enumerate(qs):
        local = 0
        for c, klo, khi in ks:
            if c != b:
                continue
            out[:, lo:hi, klo:khi] = True if on is None else on[:, i, local][:, None, None]
            local += 1
    return out


def sparse_attention(q, k, v, ok, scale):
    """o [M, H, d] and lse [H, M]; ok [H or 1, M, N]."""
    M, H, d = q.shape
    g = H // k.shape[1]
    o, lse = np.zeros((M, H, d)), np.full((H, M), -np.inf)
    for h in range(H):
        s = np.where(ok[h % len(ok)], q[:, h] @ k[:, h // g].T * scale, -np.inf)
        m = s.max(1, initial=-np.inf)
        some = m > -np.inf
        p = np.exp(s[some] - m[some, None])
        l = p.sum(1)
        o[some, h] = p @ v[:, h // g] / l[:, None]
        lse[h, some] = m[some] + np.log(l)
    return o, lse


def sparse_attention_backward(do, q, k, v, o, lse, ok, scale):
    """dq, dk, dv from the forward's o and lse."""
    H, g = q.shape[1], q.shape[1] // k.shape[1]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for h in range(H):
        j = h // g
        with np.errstate(over="ignore", invalid="ignore"):
            p = np.where(ok[h % len(ok)], np.exp(q[:, h] @ k[:, j].T * scale - lse[h][:, None]), 0.0)
        ds = p * (do[:, h] @ v[:, j].T - (do[:, h] * o[:, h]).sum(1)[:, None])
        dq[:, h] = scale * ds @ k[:, j]
        dk[:, j] += scale * ds.T @ q[:, h]
        dv[:, j] += p.T @ do[:, h]
    return dq, dk, dv

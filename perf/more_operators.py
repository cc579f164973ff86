"""The attention operators whose speed and exactness are measured, as cases.

A case is a dict of plain values; its "kind" names the operator:

  rotate      RMS norm of each head's query and key with the rotation by their
              positions (avits_qk_norm_rope)
  rotate_bwd  its backward: the gradients of the projected queries and keys and
              of the two gains (avits_qk_norm_rope_backward)
  select      which key blocks each query block attends to: the blocks' means,
              their products, the best of them (avits_block_means for queries and
              keys, avits_block_select); the means come back too
  attend      attention over the chosen blocks with its log-sum-exps
              (avits_sparse_attention)
  attend_bwd  its backward: the gradients of queries, keys and values
              (avits_sparse_attention_backward)

Sequences are text rows, then latent rows (512 text tokens with all latent tokens
at 1024^2 or 2048^2 are this repository's workloads).  Queries, keys and values are
columns of one projection's rows, [M, (H + 2 Hk) d], as a block makes them;
query head h uses key head h / (H / Hk).  Query blocks are 128 rows, key
blocks 64, counted from each sequence's first row.  A query block keeps the key
blocks that hold text rows and the `keep` others of the highest score; one that
holds text rows keeps all.  The choice is bit J % 64 of word [h, I, J / 64].
"""
import math

import torch

own = False

EPS = 1e-6
QB, KB = 128, 64


def listed():
    return [
        # One token's queries and keys: latency.
        dict(name="rotate_token", kind="rotate", dtype="bf16", M=1, H=16, Hk=16, d=128, layout="pairs", rot=128, axes=3),
        # The full grid at 2048^2, rotated by frame, row and column.
        dict(name="rotate_full_2048", kind="rotate", dtype="bf16", M=16896, H=16, Hk=16, d=128, layout="pairs", rot=128, axes=3),
        # fp32, grouped keys, part of the head in the half layout, an odd number of rows at far positions.
        dict(name="rotate_bwd_f32_odd", kind="rotate_bwd", dtype="f32", M=389, H=6, Hk=2, d=64, layout="halves", rot=44, axes=1),
        # Tuning at 1024^2.
        dict(name="rotate_bwd_1024", kind="rotate_bwd", dtype="bf16", M=4608, H=16, Hk=16, d=128, layout="pairs", rot=128, axes=3),
        # Few fp32 rows: blocks that end short.
        dict(name="select_f32_small", kind="select", dtype="f32", M=701, N=701, B=1, H=4, Hk=4, d=64, text=77, keep=3),
        # The full grid at 2048^2.
        dict(name="select_full_2048", kind="select", dtype="bf16", M=16896, N=16896, B=1, H=16, Hk=16, d=128, text=512, keep=56),
        # The fp32 exactness configuration's rows and heads.
        dict(name="attend_f32_small", kind="attend", dtype="f32", M=288, N=288, B=1, H=4, Hk=4, d=64, text=32, keep=2),
        # A single query token against the keys of a 2048^2 grid: latency and the keys' bytes.
        dict(name="attend_token", kind="attend", dtype="bf16", M=1, N=16896, B=1, H=16, Hk=4, d=128, text=512, keep=56),
        # Two images of different sizes packed one after another.
        dict(name="attend_pair", kind="attend", dtype="bf16", M=5171, N=5171, B=2, H=16, Hk=8, d=64, text=77, keep=12),
        # The full grid at 2048^2, a quarter of the keys.
        dict(name="attend_full_2048", kind="attend", dtype="bf16", M=16896, N=16896, B=1, H=16, Hk=16, d=128, text=512, keep=56),
        # A short odd sequence with grouped keys.
        dict(name="attend_bwd_small", kind="attend_bwd", dtype="bf16", M=333, N=333, B=1, H=6, Hk=2, d=64, text=40, keep=2),
        # Tuning at 1024^2 with 30 % of the keys.
        dict(name="attend_bwd_1024", kind="attend_bwd", dtype="bf16", M=4608, N=4608, B=1, H=16, Hk=16, d=128, text=512, keep=14),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate_bwd", "select", "attend", "attend", "attend_bwd", "attend_bwd"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    d = rng.choice([64, 128, 128])
    Hk = rng.choice([1, 2, 3, 4, 8, 16])
    H = Hk * rng.choice([g for g in (1, 1, 2, 3, 4, 8) if g * Hk <= 16])
    c = dict(kind=kind, dtype=dtype)
    if kind in ("rotate", "rotate_bwd"):
        rot = d if rng.random() < 0.6 else 2 * rng.randint(3, d // 2)
        return dict(c, M=_log(rng, 1, 16000 if kind == "rotate" else 4600), H=H, Hk=Hk, d=d,
                    layout=rng.choice(["pairs", "halves"]), rot=rot, axes=rng.choice([1, 3]))
    if kind == "attend" and rng.random() < 0.3:          # a few query tokens of each sequence
        B = rng.choice([1, 1, 2, 5])
        M, N = B * rng.randint(1, 4), _log(rng, 64 * B, 40000 if dtype == "bf16" else 8000)
    else:
        top = {"select": 16000, "attend": 8000, "attend_bwd": 4500}[kind] // (1 if dtype == "bf16" else 3)
        M = N = _log(rng, 1, top)
        B = rng.choice([1, 1, 2, 4])
    return dict(c, M=M, N=N, B=B, H=H, Hk=Hk, d=d, text=rng.choice([0, 40, 77, 256]), keep=rng.randint(1, 24))


def _size(c):
    return 4 if c["dtype"] == "f32" else 2


def _offsets(M, B):
    """Row offsets of B sequences of different lengths (host integers); the second of many has no rows."""
    w = [0 if B > 3 and i == 1 else 2 + 3 * i for i in range(B)]
    return [M * sum(w[:i]) // sum(w) for i in range(B)] + [M]


def _sequences(c):
    """Row offsets of the queries and of the keys."""
    k = _offsets(c["N"], c["B"])
    return (k if c["M"] == c["N"] else [c["M"] * i // c["B"] for i in range(c["B"] + 1)]), k


def _lead(c):
    """Leading rows whose query blocks keep every key block, and those whose key blocks every query block keeps."""
    return (c["text"] if c["M"] == c["N"] else 0), c["text"]


def _blocks(off, size):
    """Each sequence's first block and number of blocks."""
    n = [(b - a + size - 1) // size for a, b in zip(off, off[1:])]
    return [sum(n[:i]) for i in range(len(n) + 1)], n


# ---------------------------------------------------------------------------
# Inputs.

def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    kind, M, H, Hk, d = c["kind"], c["M"], c["H"], c["Hk"], c["d"]

    def normal(*shape, std=1.0, dtype=None):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype or dt)

    def empty(*shape, dtype=None):
        return torch.empty(*shape, device="cuda", dtype=dtype or dt)

    def columns(rows, *heads):
        """Views [rows, heads, d] of the columns of one buffer."""
        buf = rows.view(rows.shape[0], -1, d)
        return buf.split(list(heads), 1)

    s = {"case": c}
    if kind in ("rotate", "rotate_bwd"):
        rot, axes = c["rot"], c["axes"]
        dims = [rot] if axes == 1 else [rot - 4 * (rot // 6), 2 * (rot // 6), 2 * (rot // 6)]
        # The rows as the projection gives them, with a few channels ten times as large.
        x = torch.randn(M, (H + 2 * Hk) * d, generator=g, device="cuda")
        x[:, torch.randint(0, x.shape[1], (x.shape[1] // 100 + 1,), generator=g, device="cuda")] *= 10.0
        s["q"], s["k"], _ = columns(x.to(dt), H, Hk, Hk)
        s.update(g_q=1 + normal(d, std=0.2), g_k=1 + normal(d, std=0.2), dims=dims)
        if axes == 1:       # far positions of a long context
            s["pos"] = torch.randint(0, 1 << 20, (M, 1), generator=g, device="cuda", dtype=torch.int32)
            s["pos_scale"], theta = 0.25, 500000.0
        else:               # text rows at the origin, then a grid in half units
            r = (torch.arange(M, device="cuda") - min(M // 8, 512)).clamp(min=-1)
            s["pos"] = torch.stack([0 * r, 2 * (r // 128), 2 * (r % 128)], 1).clamp(min=0).to(torch.int32)
            s["pos_scale"], theta = 0.5, 10000.0
        s["freq"] = torch.cat([theta ** (-torch.arange(0, n, 2, dtype=torch.float64) / max(n, 1)) for n in dims]).cuda()
        if kind == "rotate":
            return dict(s, q_out=empty(M, H, d), k_out=empty(M, Hk, d))
        f32 = torch.float32
        s["dq"], s["dk"], _ = columns(empty(M, (H + 2 * Hk) * d), H, Hk, Hk)
        return dict(s, dq_out=normal(M, H, d, std=0.01), dk_out=normal(M, Hk, d, std=0.01), dg_q=empty(d, dtype=f32),
                    dg_k=empty(d, dtype=f32), ws=empty(64 << 20, dtype=torch.uint8))
    N = c["N"]

    def near(rows, heads):
        """Normalised, rotated heads: neighbouring rows are alike."""
        smooth = torch.randn(rows // 96 + 1, heads * d, generator=g, device="cuda")
        x = 0.8 * torch.randn(rows, heads * d, generator=g, device="cuda")
        return x + 0.6 * smooth[torch.arange(rows, device="cuda") // 96]

    if M == N:
        rows = torch.cat([near(M, H), near(M, Hk), torch.randn(M, Hk * d, generator=g, device="cuda")], 1).to(dt)
        s["q"], s["k"], s["v"] = columns(rows, H, Hk, Hk)
    else:
        s["q"] = near(M, H).to(dt).view(M, H, d)
        s["k"], s["v"] = columns(torch.cat([near(N, Hk), torch.randn(N, Hk * d, generator=g, device="cuda")], 1).to(dt), Hk, Hk)
    s["q_off"], s["k_off"] = _sequences(c)
    (_, nq), (_, nk) = _blocks(s["q_off"], QB), _blocks(s["k_off"], KB)
    words = (max(nk) + 63) // 64
    if kind == "select":
        return dict(s, q_means=empty(sum(nq), H, d, dtype=torch.float64), k_means=empty(sum(nk), Hk, d, dtype=torch.float64),
                    mask=empty(H, sum(nq), words, dtype=torch.int64))
    s["mask"] = _select(s)[2]
    s["ws"] = empty(1 << 30, dtype=torch.uint8)
    if kind == "attend":
        return dict(s, o=empty(M, H, d), lse=empty(H, M, dtype=torch.float32))
    s["o"], s["lse"] = _attend(s)
    s["do"] = normal(M, H, d, std=0.01)
    s["dq"], s["dk"], s["dv"] = columns(empty(M, (H + 2 * Hk) * d), H, Hk, Hk)
    return s


# ---------------------------------------------------------------------------
# The plain forms.

def _angles(s):
    """cos and sin [M, 1, rot / 2] of each row's pairs; the angles in 64 bits."""
    axis = torch.repeat_interleave(torch.arange(len(s["dims"]), device="cuda"),
                                   torch.tensor([n // 2 for n in s["dims"]], device="cuda"))
    a = s["pos"].double()[:, axis] * s["pos_scale"] * s["freq"]
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _turn(y, cos, sin, halves):
    """Each pair of y's leading elements turned by its angle."""
    n = 2 * cos.shape[-1]
    a, b = (y[..., :n // 2], y[..., n // 2:n]) if halves else (y[..., 0:n:2], y[..., 1:n:2])
    out = y.clone()
    if halves:
        out[..., :n // 2], out[..., n // 2:n] = a * cos - b * sin, a * sin + b * cos
    else:
        out[..., 0:n:2], out[..., 1:n:2] = a * cos - b * sin, a * sin + b * cos
    return out


def _means(x, off, size):
    """The mean of each block of rows, in 64 bits."""
    x = x.double()
    return torch.stack([x[i:min(i + size, b)].mean(0) for a, b in zip(off, off[1:]) for i in range(a, b, size)])


def _select(s):
    qm, km = _means(s["q"], s["q_off"], QB), _means(s["k"], s["k_off"], KB)
    return qm, km, _choose(s, qm, km)


def _choose(s, qm, km):
    """The mask words from the blocks' means."""
    c = s["case"]
    g = c["H"] // c["Hk"]
    q_off, k_off = s["q_off"], s["k_off"]
    (q0, nq), (k0, nk) = _blocks(q_off, QB), _blocks(k_off, KB)
    words = (max(nk) + 63) // 64
    qm, km = qm.transpose(0, 1), km.transpose(0, 1).repeat_interleave(g, 0)
    q_lead, k_lead = _lead(c)
    out = torch.zeros(c["H"], sum(nq), words, dtype=torch.int64, device="cuda")
    for b in range(c["B"]):
        if not nq[b] or not nk[b]:
            continue
        score = torch.matmul(qm[:, q0[b]:q0[b] + nq[b]], km[:, k0[b]:k0[b] + nk[b]].transpose(1, 2).contiguous())
        j = torch.arange(nk[b], device="cuda")
        lead = j * KB < k_lead
        score = torch.where(lead, -math.inf, score)
        order = torch.sort(score, dim=2, descending=True, stable=True).indices
        n = min(c["keep"], nk[b] - int(lead.sum()))
        on = torch.zeros_like(score, dtype=torch.bool).scatter_(2, order[..., :n], True) | lead
        on |= (torch.arange(nq[b], device="cuda") * QB < q_lead)[:, None]
        on = torch.nn.functional.pad(on, (0, 64 * words - nk[b])).view(*on.shape[:2], words, 64)
        out[:, q0[b]:q0[b] + nq[b]] = (on.long() << torch.arange(64, device="cuda")).sum(3)
    return out


def _allowed(s, h, b):
    """Truth values [queries, keys] of one sequence and head."""
    (q0, nq), (_, nk) = _blocks(s["q_off"], QB), _blocks(s["k_off"], KB)
    m, n = s["q_off"][b + 1] - s["q_off"][b], s["k_off"][b + 1] - s["k_off"][b]
    w = s["mask"][h, q0[b]:q0[b] + nq[b]]
    on = ((w[..., None] >> torch.arange(64, device="cuda")) & 1).bool().view(nq[b], -1)[:, :nk[b]]
    i, j = torch.arange(m, device="cuda") // QB, torch.arange(n, device="cuda") // KB
    return on[i][:, j]


def _parts(s):
    """(sequence, head, key head, query rows, key rows) of every sequence and head."""
    c = s["case"]
    for b in range(c["B"]):
        qr, kr = slice(s["q_off"][b], s["q_off"][b + 1]), slice(s["k_off"][b], s["k_off"][b + 1])
        if qr.stop > qr.start:
            for h in range(c["H"]):
                yield b, h, h // (c["H"] // c["Hk"]), qr, kr


def _attend(s):
    q, k, v, c = s["q"], s["k"], s["v"], s["case"]
    M, H, d = q.shape
    o = torch.zeros(M, H, d, dtype=q.dtype, device="cuda")
    lse = torch.full((H, M), -math.inf, device="cuda")
    for b, h, hk, qr, kr in _parts(s):
        x = (q[qr, h].float() @ k[kr, hk].float().t()) * d ** -0.5
        x = torch.where(_allowed(s, h, b), x, -math.inf)
        top = x.amax(1, keepdim=True) if x.shape[1] else torch.full((x.shape[0], 1), -math.inf, device="cuda")
        p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
        n = p.sum(1, keepdim=True)
        o[qr, h] = torch.where(n > 0, (p @ v[kr, hk].float()) / n, 0.0).to(o.dtype)
        lse[h, qr] = (top + torch.log(n))[:, 0]
    return o, lse


def _attend_bwd(s):
    q, k, v, do, c = s["q"], s["k"], s["v"], s["do"], s["case"]
    scale = c["d"] ** -0.5
    dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float32, device="cuda") for t in (q, k, v))
    for b, h, hk, qr, kr in _parts(s):
        qf, kf, vf, gf = q[qr, h].float(), k[kr, hk].float(), v[kr, hk].float(), do[qr, h].float()
        lse = s["lse"][h, qr][:, None]
        p = torch.where(_allowed(s, h, b), torch.exp(qf @ kf.t() * scale - lse), 0.0)
        ds = p * (gf @ vf.t() - (gf * s["o"][qr, h].float()).sum(1, keepdim=True)) * scale
        dq[qr, h] = ds @ kf
        dk[kr, hk] += ds.t() @ qf
        dv[kr, hk] += p.t() @ gf
    return tuple(t.to(q.dtype) for t in (dq, dk, dv))


def _plain(s):
    c, kind = s["case"], s["case"]["kind"]
    if kind == "select":
        return _select(s)
    if kind == "attend":
        return _attend(s)
    if kind == "attend_bwd":
        return _attend_bwd(s)
    cos, sin = _angles(s)
    halves = c["layout"] == "halves"
    out, gains = [], []
    for x, g, dy in ((s["q"], s["g_q"], s.get("dq_out")), (s["k"], s["g_k"], s.get("dk_out"))):
        xf, gf = x.float(), g.float()
        rstd = torch.rsqrt(xf.square().mean(2, keepdim=True) + EPS)
        n = xf * rstd
        if kind == "rotate":
            out.append(_turn(n * gf, cos, sin, halves).to(x.dtype))
            continue
        e = _turn(dy.float(), cos, -sin, halves)
        gains.append((e * n).sum((0, 1)))
        e = e * gf
        out.append((rstd * (e - n * (e * n).mean(2, keepdim=True))).to(x.dtype))
    return tuple(out + gains)


# ---------------------------------------------------------------------------
# The framework's calls.

def _own(s):
    import paper_2608_17995_amd as avits
    c, kind = s["case"], s["case"]["kind"]
    if kind in ("rotate", "rotate_bwd"):
        turn = dict(g_q=s["g_q"], g_k=s["g_k"], eps=EPS, pos=s["pos"], freq=s["freq"], dims=s["dims"], pos_scale=s["pos_scale"],
                    layout=avits.ROPE_HALVES if c["layout"] == "halves" else avits.ROPE_PAIRS)
        if kind == "rotate":
            avits.avits_qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], **turn)
            return s["q_out"], s["k_out"]
        avits.avits_qk_norm_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["dq"], s["dk"], s["dg_q"], s["dg_k"],
                                          workspace=s["ws"], **turn)
        return s["dq"], s["dk"], s["dg_q"], s["dg_k"]
    off = dict(q_off=s["q_off"], k_off=s["k_off"])
    if kind == "select":
        q_lead, k_lead = _lead(c)
        avits.avits_block_means(s["q"], QB, s["q_means"], off=s["q_off"])
        avits.avits_block_means(s["k"], KB, s["k_means"], off=s["k_off"])
        avits.avits_block_select(s["q_means"], s["k_means"], c["keep"], s["mask"], q_lead=q_lead, k_lead=k_lead, **off)
        return s["q_means"], s["k_means"], s["mask"]
    if kind == "attend":
        avits.avits_sparse_attention(s["q"], s["k"], s["v"], s["o"], mask=s["mask"], lse=s["lse"], workspace=s["ws"], **off)
        return s["o"], s["lse"]
    avits.avits_sparse_attention_backward(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["dq"], s["dk"], s["dv"],
                                          mask=s["mask"], workspace=s["ws"], **off)
    return s["dq"], s["dk"], s["dv"]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    c, kind, z = case, case["kind"], _size(case)
    M, H, Hk, d = c["M"], c["H"], c["Hk"], c["d"]
    if kind in ("rotate", "rotate_bwd"):
        n = M * (H + Hk) * d
        passes, ops = (2, 8) if kind == "rotate" else (3, 16)
        return {"bytes": passes * n * z + 4 * M * c["axes"] + 2 * d * (z + 4), "flops": ops * n}
    N = c["N"]
    q_off, k_off = _sequences(c)
    q_lead, k_lead = _lead(c)
    pairs = scores = kept = choice = 0
    for b in range(c["B"]):
        m, n = q_off[b + 1] - q_off[b], k_off[b + 1] - k_off[b]
        nk = (n + KB - 1) // KB
        lead = min(nk, (k_lead + KB - 1) // KB)
        some = min(n, KB * (lead + min(c["keep"], nk - lead)))
        full = min(m, (q_lead + QB - 1) // QB * QB)
        pairs += full * n + (m - full) * some
        kept += n if full else some if m else 0
        scores += (m + QB - 1) // QB * nk
        choice += (m + QB - 1) // QB * ((nk + 63) // 64)
    if kind == "select":
        blocks = [sum(_blocks(off, size)[1]) for off, size in ((q_off, QB), (k_off, KB))]
        return {"bytes": (M * H + N * Hk) * d * z + 8 * (blocks[0] * H + blocks[1] * Hk) * d + 8 * H * choice, "flops": (M * H + N * Hk) * d + 2 * H * scores * d}
    if kind == "attend":
        return {"bytes": (2 * M * H + 2 * kept * Hk) * d * z + 4 * H * M + 8 * H * choice, "flops": 4 * H * pairs * d}
    return {"bytes": (4 * M * H + 2 * kept * Hk + 2 * N * Hk) * d * z + 4 * H * M + 8 * H * choice, "flops": 10 * H * pairs * d}


# ---------------------------------------------------------------------------
# The definitions in 64 bits, apart from the plain forms above.

def _rotation(s):
    """Row by row the complex numbers by which the pairs are multiplied, [M, rot / 2]."""
    out, at = [], 0
    for axis, n in enumerate(s["dims"]):
        a = torch.outer(s["pos"][:, axis].double() * s["pos_scale"], s["freq"][at:at + n // 2])
        out.append(torch.polar(torch.ones_like(a), a))
        at += n // 2
    return torch.cat(out, 1)[:, None]


def _as_pairs(x, n, halves):
    return torch.complex(x[..., :n // 2], x[..., n // 2:n]) if halves else torch.view_as_complex(x[..., :n].reshape(*x.shape[:-1], n // 2, 2))


def _from_pairs(z, rest, halves):
    lead = torch.cat([z.real, z.imag], -1) if halves else torch.view_as_real(z).flatten(-2)
    return torch.cat([lead, rest], -1)


def _exact_rotate(s):
    c = s["case"]
    halves, n = c["layout"] == "halves", c["rot"]
    w = _rotation(s)
    out, gains = [], []
    for x, g, dy in ((s["q"], s["g_q"], s.get("dq_out")), (s["k"], s["g_k"], s.get("dk_out"))):
        x, g = x.double().contiguous(), g.double()
        r = ((x * x).sum(2, keepdim=True) / c["d"] + EPS) ** -0.5
        if dy is None:
            y = x * r * g
            out.append(_from_pairs(_as_pairs(y, n, halves) * w, y[..., n:], halves))
            continue
        dy = dy.double()
        e = _from_pairs(_as_pairs(dy, n, halves) * w.conj(), dy[..., n:], halves)
        gains.append((e * x * r).reshape(-1, c["d"]).sum(0))
        # d/dx of g x (avg x^2 + eps)^-1/2 against e
        out.append(e * g * r - x * r ** 3 * ((e * g * x).sum(2, keepdim=True) / c["d"]))
    return tuple(out + gains)


def _exact_select(s):
    c = s["case"]
    (q0, nq), (k0, nk) = _blocks(s["q_off"], QB), _blocks(s["k_off"], KB)
    q_lead, k_lead = _lead(c)
    words = (max(nk) + 63) // 64
    out = torch.zeros(c["H"], sum(nq), words, dtype=torch.int64)
    q_means = torch.zeros(sum(nq), c["H"], c["d"], dtype=torch.float64, device="cuda")
    k_means = torch.zeros(sum(nk), c["Hk"], c["d"], dtype=torch.float64, device="cuda")
    for b, h, hk, qr, kr in _parts(s):
        def mean(x, size):
            n = x.shape[0]
            blocks = -(-n // size)
            full = torch.zeros(blocks * size, x.shape[1], dtype=torch.float64, device="cuda")
            full[:n] = x.double()
            count = torch.full((blocks, 1), float(size), dtype=torch.float64, device="cuda")
            count[-1:] -= blocks * size - n
            return full.view(blocks, size, -1).sum(1) / count
        if kr.stop == kr.start:
            continue
        q_means[q0[b]:q0[b] + nq[b], h] = mean(s["q"][qr, h], QB)
        k_means[k0[b]:k0[b] + nk[b], hk] = mean(s["k"][kr, hk], KB)
        score = (q_means[q0[b]:q0[b] + nq[b], h] @ k_means[k0[b]:k0[b] + nk[b], hk].t()).cpu()
        first = min(nk[b], -(-k_lead // KB))
        for i in range(nq[b]):
            rest = sorted(range(first, nk[b]), key=lambda j: (-score[i, j].item(), j))[:c["keep"]] if i * QB >= q_lead else range(first, nk[b])
            for w in range(words):
                bits = sum(1 << (j - 64 * w) for j in (*range(first), *rest) if j // 64 == w)
                out[h, q0[b] + i, w] = bits - (1 << 64) if bits >> 63 else bits
    return q_means, k_means, out.cuda()


def _exact_attend(s):
    c, grads = s["case"], s["case"]["kind"] == "attend_bwd"
    M, H, d = s["q"].shape
    f64 = dict(dtype=torch.float64, device="cuda")
    o, lse = torch.zeros(M, H, d, **f64), torch.full((H, M), -math.inf, **f64)
    dq, dk, dv = (torch.zeros(s[n].shape, **f64) for n in ("q", "k", "v"))
    (q0, _), (_, nk) = _blocks(s["q_off"], QB), _blocks(s["k_off"], KB)
    for b, h, hk, qr, kr in _parts(s):
        words = s["mask"][h].cpu().tolist()
        k, v = s["k"][kr, hk].double(), s["v"][kr, hk].double()
        for i, a in enumerate(range(qr.start, qr.stop, QB)):
            r = slice(a, min(a + QB, qr.stop))
            on = [j for j in range(nk[b]) if words[q0[b] + i][j // 64] >> (j % 64) & 1]
            if not on:
                continue
            at = torch.cat([torch.arange(KB * j, min(KB * j + KB, len(k)), device="cuda") for j in on])
            q, kk, vv = s["q"][r, h].double(), k[at], v[at]
            x = q @ kk.t() / math.sqrt(d)
            if not grads:
                lse[h, r] = torch.logsumexp(x, 1)
                o[r, h] = torch.softmax(x, 1) @ vv
                continue
            p = torch.exp(x - s["lse"][h, r].double()[:, None])
            g = s["do"][r, h].double()
            e = p * (g @ vv.t() - (g * s["o"][r, h].double()).sum(1)[:, None]) / math.sqrt(d)
            dq[r, h] = e @ kk
            dk[kr, hk] = dk[kr, hk].index_add(0, at, e.t() @ q)
            dv[kr, hk] = dv[kr, hk].index_add(0, at, p.t() @ g)
    return (dq, dk, dv) if grads else (o, lse)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("rotate", "rotate_bwd"):
        return _exact_rotate(s)
    if case["kind"] == "select":
        return _exact_select(s)
    return _exact_attend(s)

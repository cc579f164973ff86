"""The low-bit and training operators whose speed and exactness are measured, as cases.

A case is a dict of plain values; its "kind" names the operator:

  norm      the modulated layer norm with the statistics its backward needs
            (avits_layer_norm)
  norm_bwd  its backward: the gradient of the rows, with the residual's added,
            and the row sums that are the gradients of scale and shift, from
            rows held in their own type or in 8 bits (avits_layer_norm_backward)
  ckpt      an activation kept in 8 bits and used in the backward pass: packed
            before the GELU, read by its gradient (avits_ckpt8_pack,
            avits_gelu_backward)
  quant     a tensor to microscaled 4-bit floats and back
            (avits_mxfp4_quantize, avits_mxfp4_dequantize)
  linear    a projection with 4-bit weights: its input quantised, then the
            product with the bias (avits_mxfp4_quantize, avits_mxfp4_linear)
  lin_bwd   the gradient of that projection's input (avits_mxfp4_linear_backward)

The rows are those of the repository's workloads (512 text tokens with 30 % of
the latent tokens at 1024^2, or with all of them at 1024^2 and 2048^2), the
widths round ones of the same order.  Hidden states are N(0, 1) about a small
mean with a few channels ten times as large, weights N(0, 0.02).

Held formats.  4-bit: codes [M, K / 2] (the low half of a byte is the even
element; bit 3 the sign, then 0, 0.5, 1, 1.5, 2, 3, 4, 6), one scale
2^(byte - 127) for 32 elements of a row, scales [ceil(K / 64), Mp, 2] with Mp
the rows rounded up to 8.  8-bit: e4m3 codes [M, D], scales [M, ceil(D / 32)].
"""
import math

import torch

own = False

EPS = 1e-6


def listed():
    return [
        # One token of the fp32 exactness configuration: latency.
        dict(name="norm_f32_token", kind="norm", dtype="f32", M=1, D=256, B=1),
        # Two images at 2048^2, each with its own modulation.
        dict(name="norm_pair_2048", kind="norm", dtype="bf16", M=33792, D=2048, B=2),
        # The compacted sequence of 1024^2 in training, rows kept as they are.
        dict(name="norm_bwd_1024", kind="norm_bwd", dtype="bf16", M=1741, D=2048, B=1, held=False),
        # A training batch of four images of different sizes, rows kept in 8 bits.
        dict(name="norm_bwd_held_batch", kind="norm_bwd", dtype="bf16", M=16901, D=4096, B=4, held=True),
        # Few fp32 rows of an odd width: blocks that end short.
        dict(name="ckpt_f32_odd", kind="ckpt", dtype="f32", M=65, D=1003),
        # The hidden layer of an MLP over the full grid at 1024^2.
        dict(name="ckpt_full_1024", kind="ckpt", dtype="bf16", M=4608, D=8192),
        # A small fp32 projection's input, a number of blocks that no vector width divides.
        dict(name="quant_f32_small", kind="quant", dtype="f32", M=37, D=1056),
        # The weight of an MLP's projection, quantised when a model is loaded.
        dict(name="quant_weight", kind="quant", dtype="bf16", M=16384, D=4096),
        # The modulation projection of one timestep: a single row.
        dict(name="linear_token", kind="linear", dtype="bf16", M=1, N=12288, K=2048),
        # An MLP's first projection over the full grid at 2048^2.
        dict(name="linear_full_2048", kind="linear", dtype="bf16", M=16896, N=8192, K=2048),
        # A few rows of the small test width.
        dict(name="lin_bwd_small", kind="lin_bwd", dtype="bf16", M=67, N=1024, K=256),
        # The same projection as above, tuned at 1024^2.
        dict(name="lin_bwd_full_1024", kind="lin_bwd", dtype="bf16", M=4608, N=8192, K=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "ckpt", "quant", "linear", "linear", "lin_bwd"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    wide = dtype == "bf16" and rng.random() < 0.7       # a width that vectors divide
    if kind in ("norm", "norm_bwd"):
        M = _log(rng, 1, 16000)
        D = 64 * _log(rng, 1, 64) if wide else _log(rng, 37, 4000)
        c = dict(kind=kind, dtype=dtype, M=M, D=D, B=rng.choice([1, 1, 2, 3, 8]))
        if kind == "norm_bwd":
            c["held"] = rng.random() < 0.5
        return c
    if kind == "ckpt":
        return dict(kind=kind, dtype=dtype, M=_log(rng, 1, 4608), D=64 * _log(rng, 1, 100) if wide else _log(rng, 37, 6000))
    if kind == "quant":
        return dict(kind=kind, dtype=dtype, M=_log(rng, 1, 16384), D=32 * _log(rng, 1, 120))
    if kind == "linear":
        return dict(kind=kind, dtype=dtype, M=_log(rng, 1, 16896), N=8 * _log(rng, 8, 1024) + rng.choice([0, 0, 0, 3]),
                    K=32 * _log(rng, 2, 64))
    return dict(kind=kind, dtype=dtype, M=_log(rng, 1, 2000 if dtype == "f32" else 4608), N=8 * _log(rng, 8, 800),
                K=32 * _log(rng, 2, 64))


def _size(c):
    return 4 if c["dtype"] == "f32" else 2


def _offsets(M, B):
    """Row offsets of B images of different sizes (host integers); the second of many has no rows."""
    if B == 1:
        return [0, M]
    w = [0 if B > 3 and i == 1 else 2 + 3 * i for i in range(B)]
    cut = [M * sum(w[:i]) // sum(w) for i in range(B)]
    return cut + [M]


# ---------------------------------------------------------------------------
# Inputs.

def _codes4(v):
    """4-bit codes of values that are on the grid (times no scale)."""
    a = v.abs()
    c = (a >= 0.5).to(torch.uint8) + (a >= 1) + (a >= 1.5) + (a >= 2) + (a >= 3) + (a >= 4) + (a >= 6)
    return c + 8 * (v < 0).to(torch.uint8)


def _hold4(w):
    """A weight in the held 4-bit form: codes [N, K / 2] and scales [ceil(K / 64), Np, 2]."""
    N, K = w.shape
    q, e = _round4(w.float())
    c = _codes4(q).view(N, K // 2, 2)
    s = torch.zeros((N + 7) // 8 * 8, (K + 63) // 64 * 2, dtype=torch.uint8, device=w.device)
    s[:N, :K // 32] = (e + 127).to(torch.uint8)
    return (c[..., 0] | (c[..., 1] << 4)).contiguous(), s.view(s.shape[0], -1, 2).permute(1, 0, 2).contiguous()


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    kind, M = c["kind"], c["M"]

    def normal(*shape, std=1.0, dtype=None):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype or dt)

    def hidden(m, d):
        x = torch.randn(m, d, generator=g, device="cuda", dtype=torch.float32) + 0.2
        x[:, torch.randint(0, d, (max(1, d // 100),), generator=g, device="cuda")] *= 10.0
        return x.to(dt)

    def empty(*shape, dtype=None):
        return torch.empty(*shape, device="cuda", dtype=dtype or dt)

    s = {"case": c}
    if kind in ("norm", "norm_bwd"):
        D, B = c["D"], c["B"]
        mod = normal(B, 6, D, std=0.3)
        s.update(off=_offsets(M, B), shift=mod[:, 3], scale=mod[:, 4])
        n = torch.tensor([b - a for a, b in zip(s["off"], s["off"][1:])], device="cuda")
        s["image"] = torch.repeat_interleave(torch.arange(B, device="cuda"), n) if B > 1 else None
        x = hidden(M, D)
        if kind == "norm":
            s.update(x=x, h=empty(M, D), mean=empty(M, dtype=torch.float32), rstd=empty(M, dtype=torch.float32))
            return s
        xf = x.double()
        mean = xf.mean(1)
        s.update(mean=mean.float(), rstd=((xf - mean[:, None]).square().mean(1) + EPS).rsqrt().float(), dh=normal(M, D, std=0.01), dres=normal(M, D, std=0.01),
                 dx=empty(M, D), dscale=empty(B, D, dtype=torch.float32), dshift=empty(B, D, dtype=torch.float32),
                 ws=empty(64 << 20, dtype=torch.uint8))
        if c["held"]:
            s["q"], s["s"] = _hold8(x)
        else:
            s["x"] = x
        return s
    if kind == "ckpt":
        D = c["D"]
        return dict(s, x=normal(M, D), da=normal(M, D, std=0.01), dm=empty(M, D), q=empty(M, D, dtype=torch.uint8),
                    s=empty(M, (D + 31) // 32, dtype=torch.uint8))
    K = c["D"] if kind == "quant" else c["K"]
    held = dict(q=empty(M, K // 2, dtype=torch.uint8), s=empty((K + 63) // 64, (M + 7) // 8 * 8, 2, dtype=torch.uint8))
    if kind == "quant":
        return dict(s, x=hidden(M, K), out=empty(M, K), **held)
    N = c["N"]
    s["wq"], s["wsc"] = _hold4(normal(N, K, std=0.02))
    s["ws"] = empty(256 << 20, dtype=torch.uint8)
    s["grid"] = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    if kind == "linear":
        return dict(s, x=hidden(M, K), b=normal(N, std=0.02), out=empty(M, N), **held)
    return dict(s, dy=normal(M, N, std=0.01), dx=empty(M, K))


# ---------------------------------------------------------------------------
# The plain forms.

def _blocks(x):
    """x [M, D] as [M, D / 32, 32], the last block filled with zeros."""
    M, D = x.shape
    n = (D + 31) // 32
    if 32 * n != D:
        x = torch.nn.functional.pad(x, (0, 32 * n - D))
    return x.view(M, n, 32)


def _round4(x):
    """fp32 rows on the 4-bit grid (times 2^exponent), and each block's exponent."""
    v = _blocks(x)
    e = torch.frexp(v.abs().amax(2)).exponent - 3       # floor(log2 of the largest) - 2
    e = torch.where(v.abs().amax(2) > 0, e, -127).clamp(-127, 125)
    y = torch.ldexp(v, -e[..., None])
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = (torch.round(a / step) * step).clamp(max=6.0)
    return torch.where(y < 0, -q, q).view(x.shape), e


def _value4(q, e):
    return torch.ldexp(_blocks(q), e[..., None]).view(q.shape)


def _read4(codes, scales, grid, M, K):
    """The values that a held 4-bit tensor stands for, in fp32."""
    c = torch.stack((codes & 15, codes >> 4), 2).view(M, K).long()
    e = scales.permute(1, 0, 2).reshape(scales.shape[1], -1)[:M, :K // 32].int() - 127
    return _value4(grid[c], e)


def _hold8(x):
    """Rows in the held 8-bit form: e4m3 codes [M, D] and scales [M, ceil(D / 32)]."""
    M, D = x.shape
    v = _blocks(x.float())
    top = torch.frexp(v.abs().amax(2))
    e = top.exponent - 9 + (top.mantissa > 0.875).int()   # the smallest power of two that leaves the largest <= 448
    e = torch.where(v.abs().amax(2) > 0, e, -127).clamp(-127, 120)
    q = torch.ldexp(v, -e[..., None]).view(M, -1)[:, :D].contiguous().to(torch.float8_e4m3fn)
    return q.view(torch.uint8), (e + 127).to(torch.uint8)


def _read8(q, s):
    M, D = q.shape
    v = torch.ldexp(_blocks(q.view(torch.float8_e4m3fn).float()), (s.int() - 127)[..., None])
    return v.view(M, -1)[:, :D]


def _images(t, image):
    """Per-image rows [B, D] spread over the images' rows, fp32 (image: each row's, or None for one image)."""
    return t.float() if image is None else t.float()[image]


def _sums(v, off):
    """The sum of each image's rows."""
    return torch.stack([v[a:b].sum(0) for a, b in zip(off, off[1:])])


def _plain(s):
    c, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        rstd = torch.rsqrt((x - mean).square().mean(1, keepdim=True) + EPS)
        h = (x - mean) * rstd * (1 + _images(s["scale"], s["image"])) + _images(s["shift"], s["image"])
        return h.to(s["x"].dtype), mean[:, 0], rstd[:, 0]
    if kind == "norm_bwd":
        x = _read8(s["q"], s["s"]) if c["held"] else s["x"].float()
        n = (x - s["mean"][:, None]) * s["rstd"][:, None]
        dh = s["dh"].float()
        gr = dh * (1 + _images(s["scale"], s["image"]))
        dx = s["rstd"][:, None] * (gr - gr.mean(1, keepdim=True) - n * (gr * n).mean(1, keepdim=True))
        return (dx + s["dres"].float()).to(s["dh"].dtype), _sums(dh * n, s["off"]), _sums(dh, s["off"])
    if kind == "ckpt":
        m = _read8(*_hold8(s["x"]))
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (m + 0.044715 * m * m * m))
        slope = 0.5 * (1 + t) + 0.5 * m * (1 - t * t) * k * (1 + 3 * 0.044715 * m * m)
        return (s["da"].float() * slope).to(s["da"].dtype)
    if kind == "quant":
        return _value4(*_round4(s["x"].float())).to(s["x"].dtype)
    w = _read4(s["wq"], s["wsc"], s["grid"], c["N"], c["K"])
    if kind == "linear":
        return (_value4(*_round4(s["x"].float())) @ w.t() + s["b"].float()).to(s["x"].dtype)
    return (s["dy"].float() @ w).to(s["dy"].dtype)


# ---------------------------------------------------------------------------
# The framework's calls.

def _own(s):
    import paper_2608_17995_amd as avits
    c, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        avits.avits_layer_norm(s["x"], s["shift"], s["scale"], s["h"], s["mean"], s["rstd"], off=s["off"], eps=EPS)
        return s["h"], s["mean"], s["rstd"]
    if kind == "norm_bwd":
        rows = dict(x_q8=s["q"], x_s8=s["s"]) if c["held"] else dict(x=s["x"])
        avits.avits_layer_norm_backward(s["dh"], s["mean"], s["rstd"], s["scale"], s["dx"], s["dscale"], s["dshift"],
                                        dres=s["dres"], off=s["off"], workspace=s["ws"], **rows)
        return s["dx"], s["dscale"], s["dshift"]
    if kind == "ckpt":
        avits.avits_ckpt8_pack(s["x"], s["q"], s["s"])
        avits.avits_gelu_backward(s["da"], s["dm"], m_q8=s["q"], m_s8=s["s"])
        return s["dm"]
    if kind == "quant":
        avits.avits_mxfp4_quantize(s["x"], s["q"], s["s"])
        avits.avits_mxfp4_dequantize(s["q"], s["s"], s["out"])
        return s["out"]
    if kind == "linear":
        avits.avits_mxfp4_quantize(s["x"], s["q"], s["s"])
        avits.avits_mxfp4_linear(s["q"], s["s"], s["wq"], s["wsc"], s["b"], s["out"], workspace=s["ws"])
        return s["out"]
    avits.avits_mxfp4_linear_backward(s["dy"], s["wq"], s["wsc"], s["dx"], workspace=s["ws"])
    return s["dx"]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    c, kind, z = case, case["kind"], _size(case)
    M = c["M"]
    if kind == "norm":
        return {"bytes": 2 * M * c["D"] * z + 8 * M + 2 * c["B"] * c["D"] * z, "flops": 8 * M * c["D"]}
    if kind == "norm_bwd":
        rows = M * c["D"] + M * ((c["D"] + 31) // 32) if c["held"] else M * c["D"] * z
        return {"bytes": 3 * M * c["D"] * z + rows + 8 * M + c["B"] * c["D"] * (z + 8), "flops": 14 * M * c["D"]}
    if kind == "ckpt":
        return {"bytes": 3 * M * c["D"] * z + 2 * (M * c["D"] + M * ((c["D"] + 31) // 32)), "flops": 24 * M * c["D"]}
    if kind == "quant":
        held = M * c["D"] // 2 + M * c["D"] // 32
        return {"bytes": 2 * M * c["D"] * z + 2 * held, "flops": 4 * M * c["D"]}
    N, K = c["N"], c["K"]
    held = N * K // 2 + N * K // 32
    return {"bytes": held + (M * K + M * N) * z + (N * z if kind == "linear" else 0), "flops": 2 * M * N * K}


# ---------------------------------------------------------------------------
# The definitions in 64 bits, apart from the plain forms above.

def _nearest(x, grid):
    """|x| to the nearest grid value, ties to the value of even index; the sign kept."""
    g = torch.tensor(grid, dtype=torch.float64, device=x.device)
    a = x.abs().clamp(max=grid[-1])
    i = torch.searchsorted(g, a.contiguous()).clamp(min=1, max=len(grid) - 1)
    lo, hi = g[i - 1], g[i]
    down, up = a - lo, hi - a
    take_hi = (up < down) | ((up == down) & (i % 2 == 0))
    return torch.where(take_hi, hi, lo) * torch.sign(x)


def _exponent(a):
    """floor(log2 a) of positive values: an estimate, put right by comparison."""
    e = torch.floor(torch.log2(a))
    e = torch.where(torch.exp2(e) > a, e - 1, e)
    return torch.where(torch.exp2(e + 1) <= a, e + 1, e)


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
_E4M3 = [i * 2.0 ** -9 for i in range(8)] + [(1 + i / 8) * 2.0 ** e for e in range(-6, 9) for i in range(8)][:-1]


def _as_held(x, grid, fit):
    """What rows stand for once held with a power-of-two scale for 32 values."""
    out = torch.empty_like(x)
    for j in range(0, x.shape[1], 32):
        v = x[:, j:j + 32]
        top = v.abs().amax(1, keepdim=True)
        e = _exponent(top.clamp(min=2.0 ** -120))
        if fit:      # the smallest scale that leaves the largest on the grid
            scale = torch.exp2(e - 8)
            scale = torch.where(top / scale > grid[-1], 2 * scale, scale)
        else:
            scale = torch.exp2(e - 2)
        out[:, j:j + 32] = torch.where(top > 0, _nearest(v / scale, grid) * scale, torch.zeros_like(v))
    return out


def _exact_read4(codes, scales, M, K):
    out = torch.empty(M, K, dtype=torch.float64, device=codes.device)
    grid = torch.tensor(_E2M1, dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        c = (codes >> (4 * half)) & 15
        out[:, half::2] = grid[(c & 7).long()] * (1.0 - 2.0 * (c >> 3).double())
    for j in range(K // 32):
        out[:, 32 * j:32 * j + 32] *= torch.exp2(scales[j // 2, :M, j % 2].double() - 127.0)[:, None]
    return out


def _exact_read8(q, s):
    grid = torch.tensor(_E4M3, dtype=torch.float64, device=q.device)
    v = grid[(q & 127).long()] * (1.0 - 2.0 * (q >> 7).double())
    for j in range(s.shape[1]):
        v[:, 32 * j:32 * j + 32] *= torch.exp2(s[:, j].double() - 127.0)[:, None]
    return v


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = case, case["kind"]
    if kind in ("norm", "norm_bwd"):
        off, D = s["off"], c["D"]
        out = []
        for b in range(c["B"]):
            r = slice(off[b], off[b + 1])
            w = 1.0 + s["scale"][b].double()
            if kind == "norm":
                x = s["x"][r].double()
                mu = x.sum(1) / D
                rs = 1.0 / torch.sqrt((x * x).sum(1) / D - mu * mu + EPS)
                out.append(((x - mu[:, None]) * rs[:, None] * w + s["shift"][b].double(), mu, rs))
                continue
            x = _exact_read8(s["q"][r], s["s"][r]) if c["held"] else s["x"][r].double()
            mu, rs, dh = s["mean"][r].double(), s["rstd"][r].double(), s["dh"][r].double()
            n = (x - mu[:, None]) * rs[:, None]
            along = ((dh * w * n).sum(1) / D)[:, None]
            level = ((dh * w).sum(1) / D)[:, None]
            out.append((s["dres"][r].double() + rs[:, None] * (dh * w - level - n * along), (dh * n).sum(0), dh.sum(0)))
        if kind == "norm":
            return tuple(torch.cat(t) for t in zip(*out))
        return torch.cat([o[0] for o in out]), torch.stack([o[1] for o in out]), torch.stack([o[2] for o in out])
    if kind == "ckpt":
        m = _as_held(s["x"].double(), _E4M3, True)
        k = math.sqrt(2.0 / math.pi)
        u = k * (m + 0.044715 * m ** 3)
        p = torch.sigmoid(2.0 * u)
        return s["da"].double() * (p + m * p * torch.sigmoid(-2.0 * u) * 2.0 * k * (1.0 + 0.134145 * m ** 2))
    if kind == "quant":
        return _as_held(s["x"].double(), _E2M1, False)
    w = _exact_read4(s["wq"], s["wsc"], c["N"], c["K"])
    if kind == "linear":
        return torch.addmm(s["b"].double(), _as_held(s["x"].double(), _E2M1, False), w.t())
    return s["dy"].double() @ w

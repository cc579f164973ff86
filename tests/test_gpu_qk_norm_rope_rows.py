"""The gains' gradients at the row counts where the backward pass shares its rows out differently, within the bound of the order
in which they are added up, and with workspaces of exactly the size."""
import numpy as np
import pytest

import oracle
from _bounds import assert_within
from test_gpu_qk_norm_rope import TURN, U, _kw, _make, _np, _other

pytestmark = pytest.mark.gpu

WAVES = 12 * 256      # the most waves of the backward pass: twelve to a CU


def _chain(M, H, Hk, d):
    """Additions that a term of a gain's gradient goes through: a lane's own (row, part) units with their steps of heads, the lanes
    of a wave, the workgroup's 8 waves, the workgroups' sums in 32 strands, the strands."""
    per_step = 64 // (d // 8)                      # heads to a step
    most = -(-max(H, Hk) // per_step)
    parts = max(1, most // 2)
    if M * parts < WAVES:
        parts = min(most, -(-WAVES // M))
    per = -(-M * parts // WAVES)
    workgroups = -(-(-(-M * parts // per)) // 8)
    return per * -(-most // parts) + per_step.bit_length() - 1 + 8 + -(-workgroups // 32) + 32


# Heads of which a row is one part, two, four (few rows), and more keys than queries.
@pytest.mark.parametrize("M,H,Hk,d", [
    (3071, 2, 1, 64), (3073, 2, 1, 64), (6145, 1, 1, 128), (1535, 16, 4, 128), (1536, 16, 4, 128), (1537, 16, 4, 128),
    (767, 16, 16, 128), (769, 16, 16, 128), (1024, 12, 12, 128), (3073, 20, 4, 128), (385, 3, 40, 64), (1, 1, 1, 64)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gain_gradients(gpu, M, H, Hk, d, dtype):
    import torch
    s = _make(M, H, Hk, d, dtype, M % 2, (d,), seed=M)
    n = gpu.avits_qk_norm_rope_backward_workspace_bytes(M, H, Hk, d)
    ws = torch.full((n + 4096,), 171, dtype=torch.uint8, device="cuda")
    dg = [torch.full((d,), 5.0, device="cuda") for _ in range(2)]
    gpu.avits_qk_norm_rope_backward(*s["dy"], *s["q"], *s["out"], *dg, workspace=ws[:n], **_kw(s))
    assert (ws[n:] == 171).all()
    with pytest.raises(gpu.AvitsError):
        gpu.avits_qk_norm_rope_backward(*s["dy"], *s["q"], *s["out"], *dg, workspace=ws[:n - 1], **_kw(s))
    ang = oracle.rope_turns(s["pos"].cpu().numpy(), s["freq"].cpu().numpy(), s["dims"], s["pos_scale"])
    for x, g, dy, got in zip(s["q"], s["g"], s["dy"], dg):
        x, dy = _np(x), _np(dy)
        _, want = oracle.norm_turn_backward(dy, x, _np(g), s["eps"], ang, bool(s["layout"]))
        e = _other(dy, sum(s["dims"]), bool(s["layout"]))
        nn = np.abs(x) / np.sqrt((x * x).mean(-1, keepdims=True) + s["eps"])
        # Each term: its turn, 14 roundings of the normalised value and the product.
        assert_within(_np(got), want, ((_chain(M, H, Hk, d) + 14) * U + TURN[dtype]) * (e * nn).sum((0, 1)), "dg")

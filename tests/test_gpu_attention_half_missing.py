"""Tensors that a call of the attention half needs and did not get are named."""
import pytest

pytestmark = pytest.mark.gpu


def test_missing(gpu):
    import torch
    q, k = (torch.zeros(9, n, 64, dtype=torch.bfloat16, device="cuda") for n in (4, 2))
    lse = torch.zeros(4, 9, device="cuda")
    turn, back = gpu.avits_qk_norm_rope, gpu.avits_qk_norm_rope_backward
    attend, attend_back = gpu.avits_sparse_attention, gpu.avits_sparse_attention_backward
    for name, call in (("q_out", lambda: turn(q, k, None, k)), ("k_out", lambda: turn(q, k, q, None)), ("k_out", lambda: turn(None, k, None, None)),
                       ("q", lambda: back(q, k, None, k, q, k)), ("k", lambda: back(q, k, q, None, q, k)), ("dq", lambda: back(q, k, q, k, None, k)),
                       ("dk", lambda: back(q, k, q, k, q, None)), ("v", lambda: attend(q, k, None, q)), ("o", lambda: attend(q, k, k, None)),
                       ("dout", lambda: attend_back(None, q, k, k, q, lse, q, k, k)), ("o", lambda: attend_back(q, q, k, k, None, lse, q, k, k)),
                       ("dv", lambda: attend_back(q, q, k, k, q, lse, q, k, None))):
        with pytest.raises(ValueError, match=f"^{name} is missing"):
            call()
    with pytest.raises(gpu.AvitsError, match="lse"):
        attend_back(q, q, k, k, q, None, q, k, k)

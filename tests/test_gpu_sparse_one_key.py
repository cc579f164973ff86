"""Sequences of one key: its probability is 1 whatever the query and the key are, so dq and dk are zero, exactly."""
import pytest

from _sparse import backward, check_backward, check_forward, forward, make

pytestmark = pytest.mark.gpu

# One row; many heads; grouped; one key under many rows (its pairs as one list, and cut into pieces); packed, some with more keys.
SHAPES = [(1, 1, 64, (0, 1), (0, 1)), (16, 16, 128, (0, 1), (0, 1)), (16, 4, 128, (0, 300), (0, 1)), (8, 2, 64, (0, 1), (0, 1)),
          (1, 1, 64, (0, 5000), (0, 1)), (6, 2, 128, (0, 200, 201, 201, 333), (0, 1, 2, 3, 4)),
          (4, 4, 64, (0, 1, 130, 135, 200), (0, 1, 66, 67, 300))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("H,Hk,d,q_off,k_off", SHAPES)
def test_one_key(gpu, H, Hk, d, q_off, k_off, dense, dtype):
    s = make(H, Hk, d, q_off, k_off, dtype, seed=61, density=0.7)
    kw = dict(mask=None) if dense else {}
    forward(gpu, s, **kw)
    check_forward(s, None if dense else "mask")
    backward(gpu, s, **kw)
    check_backward(s, None if dense else "mask")
    for qa, qb, ka, kb in zip(q_off, q_off[1:], k_off, k_off[1:]):
        if kb - ka == 1:
            assert not s["dq"][qa:qb].any() and not s["dk"][ka:kb].any()
            assert qa == qb or not dense or s["dv"][ka:kb].any()

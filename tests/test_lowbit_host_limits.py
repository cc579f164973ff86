"""The limits that the low-bit calls and their size queries share."""
import pytest

import paper_2608_17995_amd as avits

FAKE = 0x1000  # never dereferenced: every call is refused
TOP = 1 << 27


@pytest.mark.parametrize("M,K", [(TOP - 1, 1024), (TOP - 8, 576), (1 << 26, 2048), (1 << 20, 1 << 16), (8, (1 << 24) - 32), (TOP - 8, 512),
                                 (1 << 20, (1 << 16) - 64)])
def test_the_scales_query_and_the_calls_agree(M, K):
    """0 exactly where quantisation, its inverse and the products refuse the size."""
    lib = avits.load()
    size = lib.avits_mxfp4_scale_bytes(M, K)
    assert size in (0, (K + 63) // 64 * ((M + 7) // 8 * 8) * 2)
    too_many = b"2^31 scales or more"
    for refused in (lambda: lib.avits_mxfp4_quantize(None, M, K, 0, 1, None, None, None),
                    lambda: lib.avits_mxfp4_dequantize(None, None, M, K, 1, None, None)):
        assert refused() == -1 and (too_many in lib.avits_last_error()) == (size == 0)
    if K < 1 << 21:
        assert lib.avits_mxfp4_linear(None, None, M, K, FAKE, FAKE, None, 8, 1, None, None, 0, None, 1, FAKE, None, 0, None) == -1
        assert (too_many in lib.avits_last_error()) == (size == 0)
        assert (lib.avits_mxfp4_linear_backward_workspace_bytes(M, 8, K, 1) == 0) == (size == 0)

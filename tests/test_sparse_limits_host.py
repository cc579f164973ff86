"""Calls of the attention half whose workgroups would not fit a launch are refused on the host, before any device memory is touched."""
import ctypes

import pytest

import paper_2608_17995_amd as avits
from paper_2608_17995_amd import _binding as B

UNSUPPORTED = -2
FAKE, BIG = 0x1000, 1 << 62  # never dereferenced
MOST = (1 << 31) - 4097


@pytest.fixture(scope="module")
def lib():
    return avits.load()


def rows(heads):
    return ctypes.byref(B._Rows(FAKE, heads * 64))


@pytest.mark.parametrize("M,N,H,Hk,dtype", [((1 << 31) - 8192, 64, 2, 1, 1), (1 << 27, 64, 16, 16, 1), (1 << 21, 64, 1024, 1, 1), (MOST, 5, 1, 1, 0)])
def test_too_many_query_blocks(lib, M, N, H, Hk, dtype):
    q, k = rows(H), rows(Hk)
    assert lib.avits_sparse_attention(q, k, k, M, N, 1, None, None, H, Hk, 64, None, 0, 0.1, dtype, q, None, FAKE, BIG, None) == UNSUPPORTED
    assert lib.avits_sparse_attention_backward(q, q, k, k, q, FAKE, M, N, 1, None, None, H, Hk, 64, None, 0, 0.1, dtype, q, k, k, FAKE, BIG,
                                               None) == UNSUPPORTED


@pytest.mark.parametrize("N,H,dtype", [(1 << 29, 1, 1), (1 << 25, 16, 1), (MOST, 1, 0)])
def test_too_many_key_blocks(lib, N, H, dtype):
    r = rows(H)
    assert lib.avits_sparse_attention_backward(r, r, r, r, r, FAKE, 5, N, 1, None, None, H, H, 64, None, 0, 0.1, dtype, r, r, r, FAKE, BIG,
                                               None) == UNSUPPORTED


def test_too_many_choices(lib):
    assert lib.avits_block_select(FAKE, FAKE, MOST, 64 * 9000, 1, None, None, 1024, 1, 64, 0, 0, 1, FAKE, 141, None) == UNSUPPORTED

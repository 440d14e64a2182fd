"""Extents of the four-bit calls beyond what a launch holds (a grid has under 2^32 work-items): refused before anything is launched."""
import ctypes

import pytest

from paper_2504_12526_amd import binding

vp = ctypes.c_void_p
SHAPE = binding.MOM_ERR_SHAPE
A = [vp((i + 1) << 44) for i in range(10)]        # fake addresses, far apart and never dereferenced


@pytest.mark.parametrize("T", [(1 << 26) - 3, 1 << 26, 1 << 29])
def test_append_and_read_of_too_many_tokens(T):
    L = binding.lib()
    assert L.mom_mx_kv_append(None, 0, A[1], 64, A[2], 64, A[3], None, None, 0, 0, T, 0, 1, 64, None, A[4], 16, 16, None) == SHAPE
    assert L.mom_mx_kv_read(A[4], 16, 16, A[3], T, 1, 64, A[1], A[2], None) == SHAPE


@pytest.mark.parametrize("starts", [None, A[0]])
@pytest.mark.parametrize("T,B,heads,max_kv", [(1 << 21, 1 << 21, 8, 100), (1 << 20, 1 << 20, 8, 5000), (1 << 23, 1 << 23, 1, 5000), (1 << 29, 1 << 28, 2, 10)])
def test_attention_of_too_many_tiles(starts, T, B, heads, max_kv):
    assert binding.lib().mom_mx_attention(A[1], heads * 64, starts, T, B, heads, heads, 64, A[2], 16, 16, A[3], 512, A[4], max_kv, 1.0, 0, A[5], None, None, 0, None) == SHAPE


@pytest.mark.parametrize("M,N,K", [(1, 1 << 28, 32), (16, 3 << 28, 64), (1, 1 << 26, 14336), (16, 1 << 26, 32768), (16, 0x7fffff00, 4096)])
def test_products_of_too_many_rows(M, N, K):
    L = binding.lib()
    assert L.mom_mx_matvec(A[0], M, A[1], A[2], N, K, A[3], 1, None, None) == SHAPE
    assert L.mom_mx_matvec(A[0], M, A[1], A[2], N, K, A[3], 0, A[4], None) == SHAPE


@pytest.mark.parametrize("M,N,K", [(1, 1 << 27, 32), (16, 1 << 28, 64), (1, 0x7fffff00, 4096)])
def test_gate_and_up_of_too_many_rows(M, N, K):
    assert binding.lib().mom_mx_gateup(A[0], M, A[1], A[2], A[3], A[4], N, K, A[5], None) == SHAPE


@pytest.mark.parametrize("N,K", [(1 << 20, 32768), (0x7fffff00, 32), (0x7fffff00, 4096)])
def test_quantize_of_too_many_blocks(N, K):
    assert binding.lib().mom_mx_quantize(A[0], N, K, A[1], A[2], None) == SHAPE


def test_workspace_never_shrinks_with_max_kv():
    """So what a query says for max_kv is enough wherever a table holds fewer tokens."""
    wb = binding.lib().mom_mx_attention_workspace_bytes
    for T, B, q_heads, kv_heads, D in ((1, 1, 32, 8, 128), (32, 32, 32, 8, 128), (35, 7, 28, 4, 128), (64, 4, 16, 1, 64), (300, 3, 8, 2, 256), (2048, 1, 32, 8, 128), (2055, 8, 32, 8, 128),
                                       (700, 100, 16, 16, 64), (1, 1, 1, 1, 64), (5000, 2, 4, 4, 256)):
        sizes = [wb(T, B, q_heads, kv_heads, D, n) for n in [*range(0, 9000, 37), *range(9000, 1 << 20, 7001)]]
        assert sizes == sorted(sizes), (T, B, q_heads, kv_heads, D)

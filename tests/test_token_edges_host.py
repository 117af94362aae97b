"""Calls of the operators on sequences of tokens at the borders of what they take, without a GPU."""
import ctypes as C

import pytest

A = pytest.importorskip("paper_2404_09679_amd", reason="build the library first (python paper_2404_09679_amd/build.py)")
lib = A.lib
OK, INVALID = 0, -1
PTR = 1 << 20            # an address that the checks accept and nothing reads


@pytest.mark.parametrize("dtype", [0, 1])
def test_gated_backward_without_tokens_and_without_the_weights_gradients(dtype):
    """Nothing is wanted: no launch of an empty grid."""
    def bwd(N, dx, x=None):
        return lib.antdt_gated_backward(x, 16, x, 8, PTR, PTR, 16, N, 8, 16, dtype, x, dx, 8, None, None, 16, None, 0, None)

    assert bwd(0, PTR) == OK and bwd(0, None) == OK and bwd(3, None, PTR) == OK


def test_gated_block_of_more_threads_than_a_launch_has():
    """2^32 threads are the most: fp32 tiles of the forward pass are 64 x 32 by 256 threads."""
    n = C.c_size_t()
    for call in (lib.antdt_gated_forward_bytes, lib.antdt_gated_backward_bytes):
        assert call(1 << 20, 64, 32704, 0, C.byref(n)) == OK and call(1 << 20, 64, 32768, 0, C.byref(n)) == INVALID
        assert call(1 << 15, 64, (1 << 20) - 64, 0, C.byref(n)) == OK and call(1 << 16, 64, (1 << 20) - 64, 0, C.byref(n)) == INVALID
        assert call(1 << 20, 64, 32768, 1, C.byref(n)) == OK          # (bf16: larger tiles)
    assert lib.antdt_gated_saved_bytes(1 << 20, 32768, 0, C.byref(n)) == INVALID
    assert lib.antdt_gated_forward(PTR, 64, PTR, PTR, 32768, 1 << 20, 64, 32768, 0, 0, PTR, 32768, None, PTR, 1 << 30, None) == INVALID

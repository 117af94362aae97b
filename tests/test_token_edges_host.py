"""Calls of the operators on sequences of tokens at the borders of what they take, without a GPU."""
import pytest

A = pytest.importorskip("paper_2404_09679_amd", reason="build the library first (python paper_2404_09679_amd/build.py)")
lib = A.lib
OK = 0
PTR = 1 << 20            # an address that the checks accept and nothing reads


@pytest.mark.parametrize("dtype", [0, 1])
def test_gated_backward_without_tokens_and_without_the_weights_gradients(dtype):
    """Nothing is wanted: no launch of an empty grid."""
    def bwd(N, dx, x=None):
        return lib.antdt_gated_backward(x, 16, x, 8, PTR, PTR, 16, N, 8, 16, dtype, x, dx, 8, None, None, 16, None, 0, None)

    assert bwd(0, PTR) == OK and bwd(0, None) == OK and bwd(3, None, PTR) == OK

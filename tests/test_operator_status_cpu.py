"""Status calls of the operators around the layer: what is refused or reported without a GPU."""
import pytest

from paper_2503_21135_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.load()


def test_expire_linear_refusals(lib):
    """No wait to expire; otherwise what dynamo_linear_forward refuses."""
    P = 1 << 20   # an aligned address, never followed

    def call(T=40, N=8192, K=8192, G=64, ws=P, nb=1 << 30, x=P):
        return binding.STATUS_NAMES[lib.dynamo_debug_expire_linear(x, T, N, K, G, P, P, P, binding.F32, ws, nb, None)]

    assert call(T=8) == "ERR_ARG" and call(N=64) == "ERR_ARG" and call(T=0) == "ERR_ARG"
    assert call(T=-1) == "ERR_TOKENS" and call(G=32) == "ERR_SHAPE" and call(x=None) == "ERR_NULL" and call(nb=8) == "ERR_ARENA_TOO_SMALL"

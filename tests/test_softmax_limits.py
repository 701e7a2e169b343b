"""What the softmax operators refuse by size, before any device work (no GPU needed)."""
import ctypes

import pytest

UNSUPPORTED = -2
NUL, ONE = ctypes.c_void_p(0), ctypes.c_void_p(256)   # never dereferenced: validation fails first


@pytest.mark.parametrize("nb,nq,d", [(300, 1 << 30, 8), (300, 1 << 28, 65_536)])
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_gradients_of_more_tiles_than_a_launch_holds(dtype, nb, nq, d):
    import paper_2401_08281_amd as vs
    L = vs.softmax_lib()
    rc = L.vs_flat_logprob_grad(ONE, nb, ONE, nq, d, dtype, 1.0, NUL, NUL, 0, ONE, NUL, NUL, ONE, NUL, ONE, ONE, ONE, ONE, 1 << 62, NUL)
    assert rc == UNSUPPORTED and b"tiles" in L.vs_softmax_last_error()

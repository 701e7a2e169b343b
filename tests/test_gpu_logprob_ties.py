"""Equal scores go by row number, whatever the sign of a zero (GPU)."""
import pytest
import torch

from softmax_reference import INF
from test_gpu_logprob import DTYPES, check_forward, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vs():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2401_08281_amd as vs
    vs.softmax_lib()
    return vs


# kept scores, records, records beyond what a workgroup's registers hold; both sides of 16 alternatives
@pytest.mark.parametrize("nb,k", [(300, 5), (300, 40), (9001, 5), (9001, 20), (270_001, 3)])
@pytest.mark.parametrize("nq", [3, 100])
@pytest.mark.parametrize("d", [50, 64])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [0.0, -0.25])
def test_zero_scores_of_either_sign_are_equal(vs, scale, dtype, d, nq, nb, k):
    """Scores on a binary grid are exact in fp32: every score is 0 where scale is, or where the query or the row is, and a
    product of a negative scale and a zero has the other sign."""
    x, q, _, _ = make(nb, nq, d, DTYPES[dtype], 0, False, nb + nq)
    x[1::3] = 0
    x[nb // 2] = -x[nb // 2]
    q[0], q[nq // 2] = 0, 0
    check_forward(vs, x, q, None, k, scale, None)
    if scale == 0.0:
        ids = vs.vs_flat_logprob(x, q, None, k, scale=scale)[4]
        assert (ids.cpu() == torch.arange(k)).all()


@pytest.mark.parametrize("nq", [3, 100])
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_bias_of_minus_zero(vs, dtype, nq):
    x, q, _, _ = make(5000, nq, 64, DTYPES[dtype], 0, False, 7)
    x[::2] = 0
    bias = torch.zeros(5000, device="cuda")
    bias[::3] = -0.0
    bias[1::7] = -INF
    for scale in (0.0, -0.25):
        for k in (4, 30):
            check_forward(vs, x, q, None, k, scale, bias)

"""Equal scores go by row number, whatever the sign of a zero and wherever the rows lie (GPU)."""
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


@pytest.mark.parametrize("k", [3, 12, 20])
@pytest.mark.parametrize("nq", [5, 60, 100])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [100, 128])
def test_equal_rows_in_different_runs_go_by_row_number(vs, d, dtype, nq, k):
    """The same vector in several runs of 128 rows, one of which holds a second row among the best as well.  Sums of
    components between the grid's depend on their order, which must be the same for equal rows."""
    nb = 60_000
    x, q, _, _ = make(nb, nq, d, torch.float32, 0, False, 31 + d, grid=False)
    q[1:] = q[:1] * (1 + 0.003 * torch.arange(1, nq, device="cuda")[:, None])
    copies = [700, 20_001, 41_234, 59_999]
    for shift, at in enumerate(copies):
        x[at] = q[0] * 1.5
    x[705], x[41_230] = q[0] * 1.4, q[0] * 1.3                       # in the runs of the first and the third
    x, q = x.to(DTYPES[dtype]), q.to(DTYPES[dtype])
    assert all(torch.equal(x[copies[0]], x[c]) for c in copies)
    tv, ti = vs.vs_flat_logprob(x, q, None, k, scale=0.3)[3:]
    want = copies[:min(k, 4)]
    assert (ti[:, :len(want)].cpu() == torch.tensor(want)).all()
    assert (tv[:, :len(want)] == tv[:, :1]).all()
    if k > 4:
        assert (ti[:, 4].cpu() == 705).all()

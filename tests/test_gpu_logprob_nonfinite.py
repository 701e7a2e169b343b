"""Infinities and NaN among what the gradients of log-probabilities are given: rows that do not exist stay 0 (GPU)."""
import pytest
import torch

from softmax_reference import INF
from test_gpu_logprob import DTYPES, make

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def vs():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2401_08281_amd as vs
    vs.softmax_lib()
    return vs


# small tiles, large ones, products stored as they are summed and products in parts
SIZES = [("fp32", 300, 20, 33), ("bf16", 4100, 2100, 640), ("fp16", 41_000, 130, 100), ("bf16", 700, 90, 64), ("fp32", 8200, 300, 200)]


@pytest.mark.parametrize("dtype,nb,nq,d", SIZES)
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("where", ["g_logp", "g_lse", "g_entropy", "q"])
def test_rows_that_do_not_exist_have_no_gradient(vs, where, bad, dtype, nb, nq, d):
    """One query whose upstream gradient, or which itself, is not finite: its own gradient and those of the rows that exist
    are NaN, those of rows that do not exist are 0, and other queries' are as without it."""
    x, q, targets, bias = make(nb, nq, d, DTYPES[dtype], 1, True, nb + d)
    targets[:, 0] = torch.nonzero(bias > -INF)[0, 0]
    dead = bias == -INF
    x[dead] = NAN
    gl, gz, ge = (torch.full(s, 0.5, device="cuda") for s in ((nq, 1), (nq,), (nq,)))
    lse, ent = vs.vs_flat_logprob(x, q, None, 0, 0.05, bias)[1:3]
    call = lambda: vs.vs_flat_logprob_grad(x, q, lse, targets, gl, gz, ent, ge, 0.05, bias)
    dx, dq, db = call()
    assert dx.isfinite().all() and dq.isfinite().all() and (dx[dead] == 0).all() and (db[dead] == 0).all()
    i = nq // 2
    if where == "q":
        q[i, d // 2] = bad
        z = vs.vs_flat_logprob(x, q, None, 0, 0.05, bias)
        lse, ent = z[1], z[2]
    else:
        {"g_logp": gl, "g_lse": gz, "g_entropy": ge}[where][i] = bad
    ex, eq, eb = call()
    torch.cuda.synchronize()
    assert (ex[dead] == 0).all() and (eb[dead] == 0).all()
    others = torch.arange(nq, device="cuda") != i
    assert torch.equal(eq[others], dq[others])
    if where != "q":                                # (a query with an infinite component may see single rows only)
        assert eq[i].isnan().all() and ex[~dead].isnan().all() and eb[~dead].isnan().all()

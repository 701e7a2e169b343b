"""Infinite components of rows and queries that take part: an infinite score each, for few queries as for many (GPU)."""
import pytest
import torch

from softmax_reference import INF, logprob, logprob_grad, logprob_tolerance
from test_gpu_logprob import DTYPES, close, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vs():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2401_08281_amd as vs
    vs.softmax_lib()
    return vs


@pytest.mark.parametrize("dtype,d", [("fp32", 100), ("fp32", 64), ("bf16", 100), ("fp16", 100), ("bf16", 64)])
@pytest.mark.parametrize("nq", [20, 64, 65, 200])
def test_infinite_components_are_infinite_scores(vs, nq, dtype, d):
    """Rows whose score is -inf for every query weigh nothing, as the definition has it."""
    x, q, targets, bias = make(900, nq, d, DTYPES[dtype], 1, True, 5, grid=False)
    targets.clamp_(0, 899)
    q[:, 7], q[:, 40] = -q[:, 7].abs() - 0.25, q[:, 40].abs() + 0.25
    gone = torch.tensor([3, 200, 201, 640], device="cuda")
    bias[gone] = 0.5
    x[3, 7], x[200, 40], x[201, 7], x[201, 40], x[640, 7] = INF, -INF, INF, -INF, INF
    if dtype != "fp16":
        x[640, 8] = 1e30                           # finite, and beyond a smaller type's range beside an infinity
        x[640, 9] = -1e30
    lp, lse, ent, tv, ti = vs.vs_flat_logprob(x, q, targets, 5, 0.25, bias)
    without = bias.clone()
    without[gone] = -INF
    ref = logprob(x, q, targets, 5, 0.25, without)
    t, th = logprob_tolerance(ref, torch.where(x.isfinite() & (x.abs() < 1e4), x, torch.zeros_like(x)), q, 0.25, without)
    close(lse, ref["lse"], t, "lse")
    close(ent, ref["entropy"], th, "entropy")
    close(lp, ref["logp"], 2 * t, "logp")
    close(tv, ref["top_logp"], 2 * t, "top_logp")
    assert not torch.isin(ti, gone).any()
    g = -torch.ones(nq, 1, device="cuda")
    dx, dq, db = vs.vs_flat_logprob_grad(x, q, lse, targets, g, scale=0.25, bias=bias)
    hit = torch.isin(targets[:, 0], gone).any()
    assert hit or ((dx[gone] == 0).all() and (db[gone] == 0).all())
    assert db.isfinite().all() and dx.isfinite().all()
    clean = torch.where(x.isfinite() & (x.abs() < 1e4), x, torch.zeros_like(x))
    (rq, rx, rb), (tq, tx, tb) = logprob_grad(clean, q, targets, lse, None, g, None, None, 0.25, without)
    if not hit:
        close(dx, rx, tx, "dx")
        close(db, rb, tb, "dbias")


@pytest.mark.parametrize("dtype,d", [("fp32", 100), ("bf16", 100), ("bf16", 64)])
@pytest.mark.parametrize("nq", [20, 100])
def test_a_query_with_an_infinite_component(vs, nq, dtype, d):
    """Its scores are -inf where the row's component has the other sign: of 500 rows it sees none, or as many as are left."""
    x, q, _, _ = make(500, nq, d, DTYPES[dtype], 0, False, 6, grid=False)
    x[:, 4] = -x[:, 4].abs() - 0.25
    clean = vs.vs_flat_logprob(x, q, None, 3, 0.25)
    q[2, 4] = INF
    lp, lse, ent, tv, ti = vs.vs_flat_logprob(x, q, None, 3, 0.25)
    assert lse[2] == -INF and ent[2] == 0 and (tv[2] == -INF).all() and (ti[2] == -1).all()
    others = torch.arange(nq, device="cuda") != 2
    assert torch.equal(lse[others], clean[1][others]) and torch.equal(ti[others], clean[4][others])

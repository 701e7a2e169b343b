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


@pytest.mark.parametrize("dtype,d", [("fp32", 100), ("fp32", 64), ("bf16", 100), ("fp16", 33), ("fp32", 300)])
@pytest.mark.parametrize("nq", [40, 65, 300])
def test_infinities_meet(vs, nq, dtype, d):
    """One row a call, so that lse is its score: infinities of one sign stay, of both signs are NaN, as is one times zero; in the
    row, in the query, in both; NaN beside them."""
    g = torch.Generator().manual_seed(nq + d)
    q = (torch.randn(nq, d, generator=g) * 4).round() / 4
    places = torch.randint(0, d, (6,), generator=g)
    q[::5, places[0]] = INF
    q[1::7, places[1]] = -INF
    q[2::11, places[2]] = float("nan")
    for count in (0, 1, 2, 3):
        x = (torch.randn(1, d, generator=g) * 4).round() / 4
        for n in range(count):
            x[0, places[n + 1]] = INF if n % 2 == 0 else -INF
        X, Q = x.to(DTYPES[dtype]), q.to(DTYPES[dtype])
        s = (Q.double() * X.double()).sum(1) * -0.5 + 0.25
        bias = torch.full((1,), 0.25, device="cuda")
        lse = vs.vs_flat_logprob(X.cuda(), Q.cuda(), None, 0, -0.5, bias)[1].double().cpu()
        fin = s.isfinite()
        assert (lse[fin] - s[fin]).abs().max() < 1e-3 if fin.any() else True
        assert (lse[s == -INF] == -INF).all() and lse[s.isnan() | (s == INF)].isnan().all()


def test_a_table_of_infinities(vs):
    """Every row holds one, as after a diverged step: the call ends, with what is left for every query."""
    nb, nq, d = 50_000, 500, 96
    x, q, _, _ = make(nb, nq, d, torch.float32, 0, False, 9, grid=False)
    x[:, 11] = torch.where(torch.arange(nb, device="cuda") % 2 == 0, INF, -INF)
    q[:, 11] = q[:, 11].abs() + 0.25
    lse = vs.vs_flat_logprob(x, q)[1]
    assert lse.isnan().all()
    x[:, 11] = -INF
    x[nb // 2, 11] = 0.5
    lse, ent, _, ti = vs.vs_flat_logprob(x, q, None, 3)[1:]
    want = (q.double() * x[nb // 2].double()).sum(1)
    assert (lse.double() - want).abs().max() < 1e-3 and (ent == 0).all()
    assert (ti[:, 0] == nb // 2).all() and (ti[:, 1:] == -1).all()


def test_a_table_of_nan(vs):
    nb, nq, d = 50_000, 500, 96
    x, q, _, _ = make(nb, nq, d, torch.float32, 0, False, 9, grid=False)
    x[1:] = float("nan")
    lse = vs.vs_flat_logprob(x, q)[1]
    assert lse.isnan().all()
    bias = torch.full((nb,), -INF, device="cuda")
    bias[0] = 0.0
    lse = vs.vs_flat_logprob(x, q, bias=bias)[1]
    assert (lse.double() - (q.double() * x[0].double()).sum(1)).abs().max() < 1e-3

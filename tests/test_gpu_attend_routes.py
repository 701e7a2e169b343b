"""Attention over codes where the matrix cores serve it (GPU)."""
import pytest
import torch
from torch.profiler import ProfilerActivity, profile

from softmax_reference import f64
from test_gpu_attend import DTYPES, Memory

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vs():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2401_08281_amd as vs
    vs.softmax_lib()
    return vs


def by_matrix_cores(call):
    """(whether the call launches the tile kernel, what it returns)"""
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        out = call()
        torch.cuda.synchronize()
    names = [e.key for e in p.key_averages()]
    tiles, scan = (any(kind in n for n in names) for kind in ("attend_tiles_kernel", "attend_scan_kernel"))
    assert tiles != scan, names
    return tiles, out


def routes(mem, q, dk, v0):
    """Of a call and of its gradient."""
    forward, (out, lse) = by_matrix_cores(lambda: mem.ix.attend(q, 0, 0.1, v0=v0))
    back, _ = by_matrix_cores(lambda: mem.ix.attend_grad(q, 0, 0.1, lse, torch.zeros_like(out), v0=v0))
    return forward, back


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,M,dk,v0", [(128, 128, 128, 0), (96, 32, 96, 0), (256, 64, 128, 128)])
@pytest.mark.parametrize("nq", [12, 100])
def test_the_gradient_of_queries_that_see_one_row(vs, nq, d, M, dk, v0, dtype):
    """dp - mean is 0 there and g_lse k is left.  Centroid and codeword parts of sum w k and mean sum p k go through some
    sixteen fp32 operations each, of sizes up to |dp| (|c| + |t|) and |g_lse| (|c| + |t|); whatever the weights' roundings
    are, they are the same in both."""
    mt = (dk + d - v0) * M // d
    n = int((16e6 if nq <= 16 else 48e6) / (nq * mt) * 1.02) + 250
    mem = Memory(vs, n, d, M, 1, d)
    q = mem.queries(nq, dk, DTYPES[dtype])
    assert routes(mem, q, dk, v0) == (True, True)
    limits = torch.ones(nq, dtype=torch.int64)
    limits[2::3] = n                                             # (among others that see all)
    one = limits == 1
    scale = dk ** -0.5
    go, gl = torch.randn(nq, d - v0, generator=mem.g).to(q.dtype).cuda(), torch.randn(nq, generator=mem.g).cuda()
    _, lse = mem.ix.attend(q, 0, scale, v0=v0, limits=limits.cuda())
    dq = f64(mem.ix.attend_grad(q, 0, scale, lse, go, gl, v0=v0, limits=limits.cuda()))[one]
    row = mem.rows[mem.ids == 0]
    want = scale * f64(gl)[one][:, None] * row[:, :dk]
    size = f64(mem.centroids).abs().amax(0) + f64(mem.codebooks).abs().amax(1).flatten()
    dp = f64(go).abs()[one] @ size[v0:]
    tol = scale * 32 * 2.0 ** -24 * (dp + f64(gl).abs()[one])[:, None] * size[:dk] \
        + torch.finfo(q.dtype).eps / 2 * want.abs() + 2.0 ** -25
    assert ((dq - want).abs() <= tol).all(), float(((dq - want).abs() / tol).max())

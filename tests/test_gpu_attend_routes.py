"""Attention over codes: which calls the matrix cores serve, and rows around the ends of a scan's rounds (GPU)."""
import pytest
import torch
from torch.profiler import ProfilerActivity, profile

from softmax_reference import decode, f64
from test_gpu_attend import DTYPES, TILE_SHAPES, Memory, check

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


LONG = [(320, 80, 320, 0), (512, 128, 512, 0), (384, 128, 384, 0), (480, 120, 160, 160)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,M,dk,v0", [s for s in TILE_SHAPES if s[0] > 24] + LONG)
def test_calls_that_the_matrix_cores_serve(vs, d, M, dk, v0, dtype):
    """One list, 16 queries a tile and 64 (32 in the gradient), batches that end inside a tile, queries that see nothing or
    little, results of up to 512 components."""
    mt = (dk + d - v0) * M // d
    for nq in (5, 16, 17, 70, 130):
        n = int((16e6 if nq <= 16 else 48e6) / (nq * mt) * 1.02) + 250
        if max(dk, d - v0) > 256:
            n = int(48e6 / (nq * mt) * 1.02) + 250
        if n * d > 20_000_000:
            continue
        mem = Memory(vs, n, d, M, 1, nq + d)
        q = mem.queries(nq, dk, DTYPES[dtype])
        forward, back = routes(mem, q, dk, v0)
        assert forward and (back or dk > 256)         # (the gradient's tables of long keys may exceed the on-chip memory)
        check(mem, q, 0, dk, v0)
        limits = torch.randint(0, n + 1, (nq,), generator=mem.g)
        limits[0], limits[1], limits[2], limits[3] = 0, 1, -5, n // 2 // 64 * 64
        check(mem, q, 0, dk, v0, limits=limits.cuda())


@pytest.mark.parametrize("nq,n", [(1, 60_000), (3, 400_000), (16, 4000), (64, 4000)])
def test_calls_that_the_scan_serves(vs, nq, n):
    mem = Memory(vs, n, 64, 32, 1, 3)
    assert routes(mem, mem.queries(nq, 64, torch.float32), 64, 0) == (False, False)


@pytest.mark.parametrize("nq", [1, 2, 5])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("sizes", [[2040, 9], [2041, 7, 1], [2047, 1, 2048], [2048, 2048], [2056, 2040], [8, 2040, 2049], [4096, 2047, 1],
                                   [1] * 300 + [2048], [100] * 20 + [48, 1, 2000]], ids=lambda s: "-".join(map(str, s[:3])) + "+%d" % len(s))
def test_lists_that_end_at_a_round(vs, sizes, dtype, nq):
    """A round of the scan takes 2048 rows, lists padded to eight, of up to 64 lists: lists that fill one exactly, all but a
    row or a run of eight, or go on by a row."""
    g = torch.Generator().manual_seed(len(sizes))
    d, M, nlist = 32, 16, len(sizes)
    mem = Memory(vs, 0, d, M, nlist, 5, coarse=0)
    own = torch.repeat_interleave(torch.arange(nlist), torch.tensor(sizes))
    own = own[torch.randperm(own.numel(), generator=g)]
    mem.centroids = mem.centroids + torch.arange(nlist)[:, None] * 0.125          # (no two lists alike)
    mem.ix = vs.IVFPQ(d, vs.METRIC_IP, mem.centroids.cuda(), mem.codebooks.cuda(), 4)
    mem.ix.set_coarse_metric(0)
    mem.ix.add((mem.centroids[own] + torch.randn(own.numel(), d, generator=g) * 0.02).cuda())
    ids, lists = mem.ix.assignments()
    mem.ids, mem.lists = ids.cpu(), lists.long().cpu()
    mem.rows = decode(f64(mem.centroids), f64(mem.codebooks), mem.ix.codes().cpu(), mem.lists)
    q = mem.queries(nq, d, DTYPES[dtype])
    for nprobe in (0, nlist - 1 if nlist > 1 else 0):
        check(mem, q, min(nprobe, 1024), d, 0)
    check(mem, q, 0, d, 0, limits=torch.randint(0, own.numel() + 1, (nq,), generator=g).cuda())


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

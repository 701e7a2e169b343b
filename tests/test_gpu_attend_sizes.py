"""Attention over codes whose components differ in size by powers of two: results are good relative to their own
component, by the matrix cores as by the scan (GPU)."""
import pytest
import torch

from softmax_reference import HALF, INF, U, attend, decode, f64

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def vs():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2401_08281_amd as vs
    vs.softmax_lib()
    return vs


class Uneven:
    """An index whose component t is of size[t]."""

    def __init__(self, vs, n, d, M, nlist, size, seed, flat=()):
        g = torch.Generator().manual_seed(seed)
        dsub = d // M
        self.d, self.M, self.g, self.size = d, M, g, size
        self.centroids = torch.randn(nlist, d, generator=g) * size
        self.codebooks = torch.randn(M, 16, dsub, generator=g) * 0.5 * size.reshape(M, 1, dsub)
        for m in flat:                              # sub-quantizers that hold nothing
            self.codebooks[m] = 0
        own = torch.randint(0, nlist, (n,), generator=g)
        self.ix = vs.IVFPQ(d, vs.METRIC_IP, self.centroids.cuda(), self.codebooks.cuda(), 4)
        self.ix.set_coarse_metric(0)
        self.ix.add((self.centroids[own] + torch.randn(n, d, generator=g) * 0.4 * size).cuda())
        ids, lists = self.ix.assignments()
        self.rows = decode(f64(self.centroids), f64(self.codebooks), self.ix.codes().cpu(), lists.long().cpu())


def tolerances(mem, q, p, go, gl, dk, v0, scale, out, dq):
    """Every component of a stored vector, of a query and of an upstream gradient is held with an error of at most 2^-22
    relative to that component's largest codeword, and products of two such parts leave out 2^-22 again: 2^-20 of
    |q_t| max |x_t|, summed, for a score, on top of dk + M + 8 roundings of sums of these sizes in fp32 (three times: scale,
    bias and the subtraction of the maximum).  Weights: twice a score's error, and in two fp16 parts 2^-20, in one (16-bit
    queries) 2^-10 at most.  Their sums: a part of the rows (2048 at most) is taken by four wavefronts or in tiles of 64, so
    that no addition has more than 512 before it in its chain, and the parts (768 at most) by four wavefronts, another 192.
    The gradient's two sums are formed apart (sizes count)."""
    M, dt, chain = mem.M, q.dtype, 704
    rows, top = mem.rows, mem.rows.abs().amax(0)
    es = abs(scale) * (3 * (dk + M + 8) * U + 2.0 ** -20) * float((f64(q).abs() @ top[:dk]).amax())
    low = 0.0 if dt == torch.float32 else 2 * HALF[torch.float16]
    low_out = 2.0 ** -25 if dt == torch.float16 else 0.0               # steps of small fp16 results
    to = (2 * es + chain * U + 2.0 ** -20 + low) * (p @ rows[:, v0:].abs()) + 2.0 ** -22 * top[v0:] + HALF[dt] * out.abs() + low_out
    k, g = rows[:, :dk], f64(go)
    size = (g.abs() @ top[v0:])[:, None]                               # of <g, v>
    part = 4 * es + (chain + dk + M + 64) * U + 2.0 ** -19 + 2 * low
    tq = abs(scale) * part * (2 * size + gl.abs()) * (p @ k.abs() + 2.0 ** -3 * top[:dk]) + HALF[dt] * dq.abs() + low_out
    return es, to, tq


def run(vs, mem, nq, dk, v0, dtype, q_size, seed=0):
    g = mem.g
    q = torch.randn(nq, dk, generator=g) * q_size
    scale = 2.0 ** -7                              # (flat weights: the scores' error stays small beside the parts')
    q = q.to(dtype).cuda()
    go = (torch.randn(nq, mem.d - v0, generator=g) / mem.size[v0:] ** 0.5).to(dtype).cuda()
    gl = torch.randn(nq, generator=g).cuda()
    out, lse = mem.ix.attend(q, 0, scale, v0=v0)
    dq = mem.ix.attend_grad(q, 0, scale, lse, go, gl, v0=v0)
    torch.cuda.synchronize()
    ro, rl, p = attend(mem.rows, q, torch.ones(nq, mem.rows.shape[0], dtype=torch.bool), dk, v0, scale)
    k, v = mem.rows[:, :dk], mem.rows[:, v0:]
    dp = f64(go) @ v.t()
    rq = scale * ((p * (dp - (p * dp).sum(1, keepdim=True) + f64(gl)[:, None])) @ k)
    es, to, tq = tolerances(mem, q, p, go, f64(gl)[:, None], dk, v0, scale, ro, rq)
    assert es < 1e-4                                                    # (a bound that says something)
    assert ((f64(lse) - rl).abs() <= es + 704 * U + 8 * U * rl.abs().amax()).all()
    worst = ((f64(out) - ro).abs() / to).amax(0)
    assert (worst <= 1).all(), ("out", float(worst.max()), int(worst.argmax()))
    worst = ((f64(dq) - rq).abs() / tq).amax(0)
    assert (worst <= 1).all(), ("dq", float(worst.max()), int(worst.argmax()))


def steps(d, M, bits):
    """Components of every second sub-quantizer 2^-bits of the others."""
    size = torch.ones(M)
    size[1::2] = 2.0 ** -bits
    return size.repeat_interleave(d // M)


# few queries (the scan), 16 queries a tile, 64 a tile
@pytest.mark.parametrize("nq,n", [(1, 3000), (12, 60_000), (70, 30_000)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [0, 6, 10, 12, 20])
@pytest.mark.parametrize("d,M,dk,v0", [(64, 32, 64, 0), (96, 32, 48, 48), (128, 32, 128, 0)])
def test_small_sub_quantizers(vs, d, M, dk, v0, bits, dtype, nq, n):
    size = steps(d, M, bits)
    mem = Uneven(vs, n, d, M, 3, size, bits + d)
    run(vs, mem, nq, dk, v0, DTYPES[dtype], 1.0)


@pytest.mark.parametrize("nq,n", [(1, 3000), (12, 60_000), (70, 30_000)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [8, 15])
def test_queries_large_where_codewords_are_small(vs, bits, dtype, nq, n):
    """Every component weighs the same in a score: small codewords meet large queries.  (fp16 queries hold 2^15.)"""
    d, M = 64, 32
    size = steps(d, M, bits)
    mem = Uneven(vs, n, d, M, 2, size, 40 + bits)
    run(vs, mem, nq, d, 0, DTYPES[dtype], 0.5 / size)


@pytest.mark.parametrize("nq,n", [(12, 60_000), (70, 30_000)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_components_of_one_sub_quantizer_differ(vs, dtype, nq, n):
    d, M = 96, 24
    size = 2.0 ** -(torch.arange(d) % 4 * 5.0)
    mem = Uneven(vs, n, d, M, 2, size, 77)
    run(vs, mem, nq, d, 0, DTYPES[dtype], 1.0)


@pytest.mark.parametrize("nq,n", [(1, 3000), (12, 60_000), (70, 30_000)])
@pytest.mark.parametrize("centre", [1.0, 2.0 ** 20])
def test_sub_quantizers_that_hold_nothing(vs, centre, nq, n):
    """A codebook of zeros under centroids that are not: the components are the centroids', whatever their size."""
    d, M = 64, 32
    mem = Uneven(vs, n, d, M, 3, torch.full((d,), centre), 5, flat=(0, 7, 31))
    run(vs, mem, nq, d, 0, torch.float32, 1.0 / centre)
    mem = Uneven(vs, n, d, M, 3, torch.full((d,), centre), 5, flat=range(M))
    run(vs, mem, nq, d, 0, torch.float32, 1.0 / centre)

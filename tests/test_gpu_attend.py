"""Attention over the codes of a 4-bit index and its gradient on the GPU, against the definition in 64 bits
on the vectors that the index holds (read back from it: codes, lists, ids)."""
import pytest
import torch

from softmax_reference import (HALF, INF, attend, attend_grad, attend_tolerance, decode, f64, logprob, logprob_grad)

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def vs():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2401_08281_amd as vs
    vs.softmax_lib()
    return vs


class Memory:
    """An index of n vectors drawn around its centroids, and what it stores, in storage order."""

    def __init__(self, vs, n, d, M, nlist, seed, coarse=None, ids=None, size=1.0):
        g = torch.Generator().manual_seed(seed)
        self.d, self.M, self.dsub, self.nlist = d, M, d // M, nlist
        self.centroids = ((torch.randn(nlist, d, generator=g) * 8).round() / 8) * size
        self.codebooks = torch.randn(M, 16, d // M, generator=g) * 0.5 * size
        own = torch.randint(0, nlist, (n,), generator=g)
        x = self.centroids[own] + torch.randn(n, d, generator=g) * 0.4 * size
        self.ix = vs.IVFPQ(d, vs.METRIC_IP, self.centroids.cuda(), self.codebooks.cuda(), 4)
        if coarse is not None:
            self.ix.set_coarse_metric(coarse)
        if n:
            self.ix.add(x.cuda(), None if ids is None else ids.cuda())
        ids, lists = self.ix.assignments()
        self.ids, self.lists = ids.cpu(), lists.long().cpu()
        self.rows = decode(f64(self.centroids), f64(self.codebooks), self.ix.codes().cpu(), self.lists)
        self.g = g

    def queries(self, nq, dk, dtype):
        """On a grid, so that the order of the lists by their centroids does not hang on roundings."""
        q = torch.randn(nq, dk, generator=self.g)
        if self.rows.shape[0]:
            q = q + 0.7 * self.rows[torch.randint(0, self.rows.shape[0], (nq,), generator=self.g), :dk].float()
        return ((q * 16).round().clamp(-127, 127) / 16).to(dtype).cuda()

    def sees(self, q, nprobe, limits):
        nq = q.shape[0]
        out = torch.ones(nq, self.rows.shape[0], dtype=torch.bool)
        if 0 < nprobe < self.nlist:
            pad = torch.zeros(nq, self.d, device="cuda")
            pad[:, :q.shape[1]] = q
            probes = self.ix.coarse(pad, nprobe)[0].long().cpu()
            out &= (probes[:, None, :] == self.lists[None, :, None]).any(2)
        if limits is not None:
            out &= self.ids[None, :] < limits.cpu()[:, None]
        return out


def check(mem, q, nprobe, dk, v0, limits=None, scale=None, seed=0, g_lse=True):
    scale = dk ** -0.5 if scale is None else scale
    out, lse = mem.ix.attend(q, nprobe, scale, v0=v0, limits=limits)
    torch.cuda.synchronize()
    ro, rl, p = attend(mem.rows, q, mem.sees(q, nprobe, limits), dk, v0, scale)
    empty = rl == -INF
    if mem.rows.shape[0] == 0:
        assert (out == 0).all() and (lse == -INF).all()
    else:
        es, tol = attend_tolerance(mem.rows, q, p, dk, v0, scale, mem.M, q.dtype, ro)
        assert torch.equal(lse.cpu() == -INF, empty)
        big = float(rl[~empty].abs().amax()) if (~empty).any() else 0.0
        # lse: the scores' error, the sum's roundings (at most n, by some 64 in a row) and its own
        assert ((lse.double().cpu() - rl).abs()[~empty] <= es + (mem.rows.shape[0] + 64) * 2.0 ** -24 + 8 * 2.0 ** -24 * big).all()
        assert ((out.double().cpu() - ro).abs() <= tol).all(), float(((out.double().cpu() - ro).abs() - tol).max())
        assert (out.cpu()[empty] == 0).all()
    g = torch.Generator().manual_seed(seed)
    go = torch.randn(q.shape[0], mem.d - v0, generator=g).to(q.dtype).cuda()
    gl = torch.randn(q.shape[0], generator=g).cuda() if g_lse else None
    dq = mem.ix.attend_grad(q, nprobe, scale, lse, go, gl, v0=v0, limits=limits)
    torch.cuda.synchronize()
    if mem.rows.shape[0] == 0:
        assert (dq == 0).all()
        return out, lse, dq
    rq, tq = attend_grad(mem.rows, q, p, go, gl, dk, v0, scale, mem.M, es)
    assert ((dq.double().cpu() - rq).abs() <= tq).all(), float(((dq.double().cpu() - rq).abs() - tq).max())
    assert (dq.cpu()[empty] == 0).all()
    return out, lse, dq


# (d, M, dk, v0): keys that are values; keys beside values; values that are a part of the keys; sub-quantizers of one
# dimension, odd words of a code, more than 64 of them
SHAPES = [(8, 4, 8, 0), (96, 32, 96, 0), (256, 64, 128, 128), (144, 36, 144, 16), (100, 20, 100, 0), (64, 64, 32, 32),
          (6, 2, 6, 3), (160, 80, 160, 0), (24, 6, 8, 12), (128, 128, 128, 0), (512, 64, 256, 256), (768, 64, 768, 0)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,M,dk,v0", SHAPES)
def test_all_lists(vs, dtype, d, M, dk, v0):
    for n, nlist, nq in ((1, 1, 1), (63, 5, 2), (1500, 1, 9), (4000, 70, 33)):
        mem = Memory(vs, n, d, M, nlist, n + d)
        check(mem, mem.queries(nq, dk, DTYPES[dtype]), 0, dk, v0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,M,dk,v0", SHAPES)
@pytest.mark.parametrize("coarse", [0, 1])
def test_probed_lists(vs, dtype, d, M, dk, v0, coarse):
    mem = Memory(vs, 3000, d, M, 40, 7 + d, coarse=coarse)
    for nq, nprobe in ((1, 1), (3, 7), (40, 39), (2, 40)):
        check(mem, mem.queries(nq, dk, DTYPES[dtype]), nprobe, dk, v0)


def codes_for_tiles(nq, mt, nlist_of=None, least=None):
    """Stored vectors from which on nq queries go through the matrix cores (mt: look-ups a pair)."""
    least = (16e6 if nq <= 16 else 48e6) if least is None else least
    return int(least * (1 if nlist_of is None else 1 + 100.0 / (nlist_of - 8)) / (nq * mt)) + 77


TILE_SHAPES = [s for s in SHAPES if s[0] != 768] + [(66, 22, 66, 0), (140, 28, 140, 5), (258, 86, 129, 129), (130, 26, 65, 65)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,M,dk,v0", TILE_SHAPES)
def test_many_queries(vs, dtype, d, M, dk, v0):
    """Enough work for the matrix cores: 16 queries a tile and 64, one list and lists of 90, some queries that see
    nothing or little, a batch that ends inside a tile."""
    mt = (dk + d - v0) * M // d
    for nq, run in ((5, None), (16, 90), (17, None), (65, 90), (130, None)):
        n = codes_for_tiles(nq, mt, run)
        if n > 400_000 or n * d > 20_000_000:
            continue
        mem = Memory(vs, n, d, M, 1 if run is None else n // run, nq + d)
        q = mem.queries(nq, dk, DTYPES[dtype])
        check(mem, q, 0, dk, v0)
        limits = torch.randint(0, n + 1, (nq,), generator=mem.g)
        limits[0], limits[1], limits[2], limits[3] = 0, 1, -5, n // 2 // 64 * 64
        check(mem, q, 0, dk, v0, limits=limits.cuda())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,M,dk,v0,nq,least", [(320, 80, 320, 0, 20, 48e6), (384, 64, 66, 0, 70, 256e6), (512, 128, 512, 0, 16, 48e6)])
def test_long_results(vs, dtype, d, M, dk, v0, nq, least):
    mem = Memory(vs, codes_for_tiles(nq, (dk + d - v0) * M // d, None, least), d, M, 1, d)
    check(mem, mem.queries(nq, dk, DTYPES[dtype]), 0, dk, v0)


@pytest.mark.parametrize("nq", [16, 100])
def test_many_queries_on_lists_of_all_lengths(vs, nq):
    """Lists that are empty, of one vector, of a tile and one more or less, among long ones; ids in another order."""
    g = torch.Generator().manual_seed(15)
    d, M, nlist = 32, 16, 200
    sizes = [25000, 0, 1, 0, 0, 63, 64, 65, 128, 30000, 2049] + [int(v) for v in torch.randint(0, 130, (nlist - 11,), generator=g)]
    own = torch.repeat_interleave(torch.arange(nlist), torch.tensor(sizes))
    own = own[torch.randperm(own.numel(), generator=g)]
    mem = Memory(vs, 0, d, M, nlist, 5, coarse=0)
    ids = torch.randperm(own.numel(), generator=g)
    mem.ix.add((mem.centroids[own] + torch.randn(own.numel(), d, generator=g) * 0.05).cuda(), ids.cuda())
    got, lists = mem.ix.assignments()
    mem.ids, mem.lists = got.cpu(), lists.long().cpu()
    mem.rows = decode(f64(mem.centroids), f64(mem.codebooks), mem.ix.codes().cpu(), mem.lists)
    q = mem.queries(nq, d, torch.float32)
    check(mem, q, 0, d, 0)
    check(mem, q, 0, d, 0, limits=torch.randint(0, own.numel(), (nq,), generator=g).cuda())
    check(mem, q, 0, d, 0, limits=torch.full((nq,), 3).cuda())


@pytest.mark.parametrize("scale", [0.0, -0.3, 40.0])
def test_many_queries_flat_and_sharp(vs, scale):
    mem = Memory(vs, 12_000, 64, 32, 3, 8)
    check(mem, mem.queries(70, 64, torch.float32), 0, 64, 0, scale=scale)


@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** 20])
def test_many_queries_magnitudes(vs, size):
    mem = Memory(vs, 25_000, 32, 16, 2, 9, size=size)
    q = (mem.queries(64, 32, torch.float32).clamp(-8, 8) / size).contiguous()
    out, lse = mem.ix.attend(q, 0, 0.1)
    ro, rl, p = attend(mem.rows, q, mem.sees(q, 0, None), 32, 0, 0.1)
    es, tol = attend_tolerance(mem.rows / size, q * size, p, 32, 0, 0.1, mem.M, q.dtype, ro / size)
    assert ((out.double().cpu() - ro).abs() / size <= tol).all()
    assert ((lse.double().cpu() - rl).abs() <= es + 25_064 * 2.0 ** -24 + 2.0 ** -20 * float(rl.abs().amax())).all()


@pytest.mark.parametrize("nprobe", [0, 5])
@pytest.mark.parametrize("nq", [1, 2, 17, 130])
@pytest.mark.parametrize("dtype", DTYPES)
def test_limits(vs, nprobe, nq, dtype):
    """Positions up to a query's own; queries that see one vector, or none, among others."""
    mem = Memory(vs, 2500, 64, 32, 30 if nprobe else 1, 3)
    q = mem.queries(nq, 32, DTYPES[dtype])
    limits = torch.randint(0, 2501, (nq,), generator=mem.g)
    limits[0] = 0
    if nq > 2:
        limits[1], limits[2] = 1, -5
    if nq > 5:
        limits[3], limits[4], limits[5] = 2500, 1 << 40, 64
    check(mem, q, nprobe, 32, 32, limits=limits.cuda())
    check(mem, q, nprobe, 32, 32, limits=torch.zeros_like(limits).cuda())


def test_ids_decide_about_limits_not_places(vs):
    n = 900
    ids = torch.randperm(n, generator=torch.Generator().manual_seed(1)) * 5_000_000_000
    mem = Memory(vs, n, 32, 16, 12, 4, ids=ids)
    q = mem.queries(20, 32, torch.float32)
    limits = torch.randint(0, n, (20,), generator=mem.g) * 5_000_000_000
    check(mem, q, 0, 32, 0, limits=limits.cuda())
    check(mem, q, 4, 32, 0, limits=limits.cuda())


@pytest.mark.parametrize("nq", [1, 20])
def test_lists_of_all_lengths(vs, nq):
    """A long list (several rounds of 1024), empty ones, lists of one vector, and more lists than a round takes."""
    g = torch.Generator().manual_seed(5)
    d, M, nlist = 32, 16, 300
    mem = Memory(vs, 0, d, M, nlist, 5, coarse=0)
    sizes = [5000, 0, 1, 0, 0, 63, 64, 65, 1024, 1, 2049] + [int(v) for v in torch.randint(0, 4, (nlist - 11,), generator=g)]
    own = torch.repeat_interleave(torch.arange(nlist), torch.tensor(sizes))
    own = own[torch.randperm(own.numel(), generator=g)]
    mem.ix.add((mem.centroids[own] + torch.randn(own.numel(), d, generator=g) * 0.05).cuda())
    ids, lists = mem.ix.assignments()
    mem.ids, mem.lists = ids.cpu(), lists.long().cpu()
    mem.rows = decode(f64(mem.centroids), f64(mem.codebooks), mem.ix.codes().cpu(), mem.lists)
    q = mem.queries(nq, d, torch.float32)
    for nprobe in (0, 1, 100, 299):
        check(mem, q, nprobe, d, 0)


@pytest.mark.parametrize("nq", [1, 3, 40])
def test_empty_index(vs, nq):
    mem = Memory(vs, 0, 16, 8, 10, 6)
    q = mem.queries(nq, 16, torch.float32)
    check(mem, q, 0, 16, 0)
    check(mem, q, 3, 16, 0)


@pytest.mark.parametrize("nq", [1, 40])
@pytest.mark.parametrize("scale", [0.0, -0.3, 40.0])
def test_flat_and_sharp_weights(vs, nq, scale):
    mem = Memory(vs, 3000, 64, 32, 3, 8)
    check(mem, mem.queries(nq, 64, torch.float32), 0, 64, 0, scale=scale)


@pytest.mark.parametrize("nq", [1, 64])
@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** 20])
def test_magnitudes(vs, nq, size):
    mem = Memory(vs, 1500, 32, 16, 2, 9, size=size)
    q = (mem.queries(nq, 32, torch.float32).clamp(-8, 8) / size).contiguous()
    out, lse = mem.ix.attend(q, 0, 0.1)
    ro, rl, p = attend(mem.rows, q, mem.sees(q, 0, None), 32, 0, 0.1)
    es, tol = attend_tolerance(mem.rows / size, q * size, p, 32, 0, 0.1, mem.M, q.dtype, ro / size)
    assert ((out.double().cpu() - ro).abs() / size <= tol).all()
    assert ((lse.double().cpu() - rl).abs() <= es + 2000 * 2.0 ** -24 + 2.0 ** -20 * float(rl.abs().amax())).all()


def test_gradient_agrees_with_differences(vs):
    mem = Memory(vs, 700, 48, 24, 5, 10)
    q = mem.queries(6, 32, torch.float32)
    g = torch.Generator().manual_seed(2)
    go, gl, u = torch.randn(6, 32, generator=g), torch.randn(6, generator=g), torch.randn(6, 32, generator=g, dtype=torch.float64)
    _, lse = mem.ix.attend(q, 0, 0.2, v0=16)
    dq = mem.ix.attend_grad(q, 0, 0.2, lse, go.cuda(), gl.cuda(), v0=16)

    def loss(qd):
        o, z, _ = attend(mem.rows, qd, torch.ones(6, 700, dtype=torch.bool), 32, 16, 0.2)
        return (o * go.double()).sum() + (z * gl.double()).sum()

    e = 1e-4
    along = (loss(f64(q) + e * u) - loss(f64(q) - e * u)) / (2 * e)
    inner = f64(dq) * u
    assert abs(along - inner.sum()) <= 1e-5 * inner.abs().sum()


def test_equal_calls_give_equal_bits_on_any_stream(vs):
    mem = Memory(vs, 9000, 128, 32, 50, 11)
    for nq, nprobe, dtype in ((1, 0, "fp32"), (100, 0, "bf16"), (200, 0, "fp32"), (100, 8, "fp32")):
        q = mem.queries(nq, 128, DTYPES[dtype])
        go = torch.randn(nq, 128, device="cuda").to(q.dtype)
        run = lambda: mem.ix.attend(q, nprobe, 0.1)
        a = run()
        da = mem.ix.attend_grad(q, nprobe, 0.1, a[1], go)
        torch.cuda.synchronize()
        outs = []
        for st in [torch.cuda.Stream() for _ in range(2)]:
            with torch.cuda.stream(st):
                b = run()
                outs.append(b + (mem.ix.attend_grad(q, nprobe, 0.1, b[1], go),))
        torch.cuda.synchronize()
        for o in outs:
            for u, v in zip(a + (da,), o):
                assert torch.equal(u, v)


@pytest.mark.parametrize("nq,n", [(1, 4000), (40, 4000), (40, 20_000)])
def test_captured_and_replayed(vs, nq, n):
    mem = Memory(vs, n, 64, 32, 20, 12)
    q = mem.queries(nq, 64, torch.bfloat16)
    go = torch.randn(nq, 64, device="cuda").bfloat16()
    limits = torch.full((nq,), 3000, device="cuda")

    def both():
        o, z = mem.ix.attend(q, 0, 0.1, limits=limits)
        return o, z, mem.ix.attend_grad(q, 0, 0.1, z, go, limits=limits)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for r in range(4):
        q.copy_(mem.queries(nq, 64, torch.bfloat16))
        limits.fill_(500 * r)
        want = [t.clone() for t in both()]
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(out, want):
            assert torch.equal(u, v)


def test_probed_lists_are_refused_under_capture(vs):
    """The coarse quantizer's work space is the index's own: a replay could meet it at another size or in use."""
    mem = Memory(vs, 1000, 64, 32, 20, 12)
    q = mem.queries(4, 64, torch.float32)
    want = mem.ix.attend(q, 5, 0.1)
    go = torch.ones_like(q)
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        for call in (lambda: mem.ix.attend(q, 5, 0.1), lambda: mem.ix.attend_grad(q, 5, 0.1, want[1], go)):
            with pytest.raises(vs.VSError) as e:
                call()
            assert e.value.code == -2
        all_lists = mem.ix.attend(q, 20, 0.1)
    assert all_lists[0].shape == q.shape
    for u, v in zip(want, mem.ix.attend(q, 5, 0.1)):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq,n,nprobe", [(2, 500, 0), (10, 4000, 3), (16, 30_000, 0), (70, 20_000, 0)])
def test_padded_queries(vs, dtype, nq, n, nprobe):
    """Queries of a batch that are padding, with a limit of 0 and anything inside, answer with zeros, and the others as
    they do without them; a NaN query that sees rows does not reach the others either."""
    mem = Memory(vs, n, 64, 32, 6, 17)
    q = mem.queries(nq, 64, DTYPES[dtype])
    limits = torch.full((nq,), n)
    pad = torch.arange(1, nq, 3)
    limits[pad] = 0
    go = torch.randn(nq, 64, generator=mem.g).to(q.dtype).cuda()
    gl = torch.randn(nq, generator=mem.g).cuda()
    q[pad], go[pad] = 0, 0
    out, lse = mem.ix.attend(q, nprobe, 0.1, limits=limits.cuda())
    dq = mem.ix.attend_grad(q, nprobe, 0.1, lse, go, gl, limits=limits.cuda())
    for bad in (float("nan"), INF, -INF, float(torch.finfo(q.dtype).max)):
        q[pad], go[pad], gl[pad] = bad, bad, bad
        o2, z2 = mem.ix.attend(q, nprobe, 0.1, limits=limits.cuda())
        d2 = mem.ix.attend_grad(q, nprobe, 0.1, z2, go, gl, limits=limits.cuda())
        assert (z2[pad] == -INF).all() and (o2[pad] == 0).all() and (d2[pad] == 0).all()
        assert torch.equal(o2, out) and torch.equal(z2, lse) and torch.equal(d2, dq)
    q[pad] = float("nan")
    o2, z2 = mem.ix.attend(q, nprobe, 0.1)
    live = torch.ones(nq, dtype=torch.bool)
    live[pad] = False
    assert torch.equal(o2[live], out[live]) and torch.equal(z2[live], lse[live])
    if nprobe == 0:
        assert z2[pad].isnan().all() and o2[pad].isnan().all()


def test_search_and_attention_share_an_index(vs):
    """Attention leaves the index as it is, and a growing index is attended as it stands."""
    mem = Memory(vs, 2000, 64, 32, 16, 13)
    q = mem.queries(30, 64, torch.float32)
    before = mem.ix.search(q, 10, 4)
    mem.ix.attend(q, 4, 0.1)
    mem.ix.attend(q, 0, 0.1)
    for u, v in zip(before, mem.ix.search(q, 10, 4)):
        assert torch.equal(u, v)
    # sharp weights: the heaviest vector is the best one of a search over all lists
    D, I = mem.ix.search(q, 1, 16)
    _, lse = mem.ix.attend(q, 0, 64.0)
    assert ((lse / 64.0 - D[:, 0]).abs() <= 1e-4 * D[:, 0].abs() + 0.12).all()      # log(2000) / 64 at most above it
    more = torch.randn(500, 64, generator=mem.g)
    mem.ix.add(more.cuda())
    ids, lists = mem.ix.assignments()
    mem.ids, mem.lists = ids.cpu(), lists.long().cpu()
    mem.rows = decode(f64(mem.centroids), f64(mem.codebooks), mem.ix.codes().cpu(), mem.lists)
    assert mem.rows.shape[0] == 2500
    check(mem, q, 0, 64, 0)


def test_memory_then_log_probabilities_and_back(vs):
    """The operators as they are used together: a hidden state reads a compressed memory, the sum is scored against a
    table of embeddings, and the loss goes back through both to the state and the table."""
    mem = Memory(vs, 3000, 128, 32, 1, 14)
    g = torch.Generator().manual_seed(4)
    nq, nb = 70, 900
    h = mem.queries(nq, 64, torch.float32)
    x = torch.randn(nb, 64, generator=g).cuda()
    targets = torch.randint(0, nb, (nq, 1), generator=g).cuda()
    limits = torch.randint(1, 3001, (nq,), generator=g).cuda()
    out, z = mem.ix.attend(h, 0, 0.125, v0=64, limits=limits)
    y = (h + out).contiguous()
    logp, lse, ent, _, _ = vs.vs_flat_logprob(x, y, targets, 0, 0.125)
    gl = torch.full((nq, 1), -1.0 / nq, device="cuda")
    dx, dy, _ = vs.vs_flat_logprob_grad(x, y, lse, targets, gl, scale=0.125)
    dh = dy + mem.ix.attend_grad(h, 0, 0.125, z, dy, v0=64, limits=limits)
    hd, xd = f64(h).requires_grad_(), f64(x).requires_grad_()
    s = 0.125 * hd @ mem.rows[:, :64].t()
    s = torch.where(mem.sees(h, 0, limits), s, torch.full_like(s, -INF))
    o = torch.softmax(s, 1) @ mem.rows[:, 64:]
    loss = -torch.log_softmax(0.125 * (hd + o) @ xd.t(), 1).gather(1, targets.cpu()).mean()
    loss.backward()
    assert abs(-logp.double().mean().cpu() - loss) < 1e-5 * loss
    # every step is good to some 1e-5 of the sizes that enter it (the tests above); a softmax passes errors on at most doubled
    for got, want in ((dh, hd.grad), (dx, xd.grad)):
        assert (f64(got) - want).abs().max() <= 1e-4 * want.abs().max()


def test_refusals(vs):
    mem = Memory(vs, 200, 32, 8, 4, 15)
    q = mem.queries(3, 32, torch.float32)
    for kw in (dict(v0=-4), dict(v0=32), dict(v0=2)):
        with pytest.raises((vs.VSError, ValueError)):
            mem.ix.attend(q, 0, 1.0, **kw)
    for bad in (q[:, :30].contiguous(), torch.zeros(3, 36, device="cuda")):
        with pytest.raises(vs.VSError):
            mem.ix.attend(bad, 0, 1.0)
    for nprobe in (-1, 1025):
        with pytest.raises(vs.VSError):
            mem.ix.attend(q, nprobe, 1.0)
    with pytest.raises(vs.VSError):
        mem.ix.attend(q, 0, float("nan"))
    with pytest.raises(TypeError):
        mem.ix.attend(q.double(), 0, 1.0)
    with pytest.raises(TypeError):
        mem.ix.attend(q, 0, 1.0, limits=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        mem.ix.attend(q, 0, 1.0, limits=torch.zeros(2, dtype=torch.int64, device="cuda"))
    lse = mem.ix.attend(q, 0, 1.0)[1]
    with pytest.raises(ValueError):
        mem.ix.attend_grad(q, 0, 1.0, lse, torch.zeros(3, 31, device="cuda"))
    with pytest.raises(TypeError):
        mem.ix.attend_grad(q, 0, 1.0, lse, torch.zeros(3, 32, device="cuda").half())
    t = lambda *s: torch.randn(*s, device="cuda")
    for ix in (vs.IVFPQ(32, vs.METRIC_L2, t(4, 32), t(8, 16, 4), 4), vs.IVFPQ(32, vs.METRIC_IP, t(4, 32), t(8, 256, 4), 8),
               vs.IVFPQ(1024, vs.METRIC_IP, t(2, 1024), t(1024, 16, 1), 4)):
        with pytest.raises(vs.VSError) as e:
            ix.attend(t(2, ix.d), 0, 1.0)
        assert e.value.code == -2
    # a work space that is too small
    L = vs.softmax_lib()
    import ctypes
    p = lambda x: ctypes.c_void_p(x.data_ptr())
    out, z, ws = torch.empty_like(q), torch.empty(3, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    need = vs.vs_ivfpq_attend_workspace_bytes(mem.ix.h, 3, 32, 0, 0, 0)
    assert L.vs_ivfpq_attend(mem.ix.h, p(q), 3, 32, 0, 0, 0, 1.0, None, p(out), p(z), p(ws), need - 1, None) == -1
    assert b"work space" in L.vs_softmax_last_error()
    empty = mem.ix.attend(q[:0], 0, 1.0)
    assert empty[0].shape == (0, 32) and empty[1].shape == (0,)

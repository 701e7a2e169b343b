"""Log-probabilities over rows and their gradients on the GPU, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from softmax_reference import INF, logprob, logprob_grad, logprob_tolerance

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def vs():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2401_08281_amd as vs
    vs.softmax_lib()
    return vs


def make(nb, nq, d, dtype, nt, masked, seed, grid=True):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(nb, d, generator=g) * 32).round().clamp(-127, 127) / 64
    q = (torch.randn(nq, d, generator=g) * 32).round().clamp(-127, 127) / 64
    if not grid:
        x, q = x + 0.003 * torch.randn(nb, d, generator=g), q + 0.003 * torch.randn(nq, d, generator=g)
    bias = None
    if masked:
        bias = (torch.randn(nb, generator=g) * 32).round() / 64
        bias[torch.rand(nb, generator=g) < 0.2] = -INF
    targets = torch.randint(-2, nb + 2, (nq, nt), generator=g) if nt else None
    dev = lambda t: None if t is None else t.cuda()
    return x.to(dtype).cuda(), q.to(dtype).cuda(), dev(targets), dev(bias)


def close(got, want, tol, what):
    got, want = got.double().cpu(), want.double()
    fin = want.isfinite()
    assert torch.equal(got[~fin], want[~fin]), what
    worst = ((got - want).abs() - tol)[fin] if isinstance(tol, float) else (got - want).abs()[fin] - tol[fin]
    assert got[fin].isfinite().all() and (worst.numel() == 0 or worst.max() <= 0), (what, float(worst.max()))


def check_forward(vs, x, q, targets, k, scale, bias):
    lp, lse, ent, tv, ti = vs.vs_flat_logprob(x, q, targets, k, scale=scale, bias=bias)
    torch.cuda.synchronize()
    ref = logprob(x, q, targets, k, scale, bias)
    t, th = logprob_tolerance(ref, x, q, scale, bias)
    close(lse, ref["lse"], t, "lse")
    close(ent, ref["entropy"], th, "entropy")
    if targets is not None:
        close(lp, ref["logp"], 2 * t, "logp")
    if k:
        assert torch.equal(ti.cpu(), ref["top_ids"])
        close(tv, ref["top_logp"], 2 * t, "top_logp")
    return lse, ent


# every route: up to 16, 32, 64 queries and more; dimensions of whole blocks and ragged ones, odd ones (rows that start
# anywhere); kept scores (few records for the k) and records; records that hold several of the best
SHAPES = [(1, 1, 1, 1), (2, 1, 7, 3), (129, 3, 33, 5), (500, 16, 128, 10), (1000, 17, 100, 1), (3000, 33, 65, 64),
          (20_000, 5, 768, 3), (40_000, 64, 48, 40), (127, 65, 64, 5), (128, 128, 256, 0), (129, 129, 31, 2),
          (5000, 300, 96, 9), (60_001, 130, 64, 7), (300, 70, 1030, 4), (100_000, 5, 64, 20), (30_000, 33, 128, 17),
          (2000, 32, 320, 5), (2100, 33, 320, 5), (2000, 64, 100, 40), (257, 256, 64, 64)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nb,nq,d,k", SHAPES)
@pytest.mark.parametrize("masked", [False, True])
def test_forward(vs, dtype, nb, nq, d, k, masked):
    x, q, targets, bias = make(nb, nq, d, DTYPES[dtype], 3, masked, nb + nq)
    check_forward(vs, x, q, targets, k, 0.25, bias)


def test_best_rows_share_a_record(vs):
    """All of the k best lie in one run of 128 rows, and equal scores go by row number."""
    nb, d = 50_000, 64
    x, q, _, _ = make(nb, 70, d, torch.float32, 0, False, 5)
    q[:] = q[:1]
    for j in (40_003, 40_001, 40_100, 40_002, 12, 49_999):
        x[j] = q[0] * 1.5
    for n in (3, 70):
        _, ids = vs.vs_flat_logprob(x, q[:n].contiguous(), None, 8, scale=0.25)[3:]
        assert (ids[:, :6].cpu() == torch.tensor([12, 40_001, 40_002, 40_003, 40_100, 49_999])).all()
        check_forward(vs, x, q[:n].contiguous(), None, 8, 0.25, None)


@pytest.mark.parametrize("nq", [1, 20, 40, 100])
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_do_not_exist(vs, nq, dtype):
    """Rows with a bias of -inf count nowhere, whatever they hold; without any other row the results are empty."""
    x, q, targets, bias = make(700, nq, 64, DTYPES[dtype], 2, True, 3)
    dead = bias == -INF
    x[dead] = float("nan")
    x[dead.nonzero()[0, 0]] = INF
    lse, ent = check_forward(vs, x, q, targets, 6, 0.25, bias)
    check_grad(vs, x, q, targets, lse, ent, 0.25, bias, 1)
    gone = torch.full_like(bias, -INF)
    lp, lse, ent, tv, ti = vs.vs_flat_logprob(x, q, targets, 6, bias=gone)
    assert (lse == -INF).all() and (ent == 0).all() and (tv == -INF).all() and (ti == -1).all()
    ok = (targets >= 0) & (targets < 700)
    assert (lp[ok] == -INF).all() and (lp[~ok] == 0).all()
    dx, dq, db = vs.vs_flat_logprob_grad(x, q, lse, targets, torch.ones_like(lp), bias=gone)
    assert (dx == 0).all() and (dq == 0).all() and (db == 0).all()


@pytest.mark.parametrize("nq", [3, 100])
def test_lowest_bias_is_a_score_like_others(vs, nq):
    x, q, _, _ = make(300, nq, 32, torch.float32, 0, False, 4)
    low = torch.finfo(torch.float32).min
    bias = torch.full((300,), low, device="cuda")
    lse = vs.vs_flat_logprob(x, q, bias=bias)[1]
    # scores vanish in the roundings of the bias: 300 equal ones (whose logarithm vanishes as well)
    assert (lse == low).all()
    bias[7] = 0.0
    _, lse, ent, tv, ti = vs.vs_flat_logprob(x, q, None, 2, scale=0.5, bias=bias)
    want = 0.5 * (q.double() @ x[7].double())
    assert (lse.double() - want).abs().max() < 1e-5 and (ent == 0).all() and (ti[:, 0] == 7).all() and (tv[:, 0] == 0).all()


def test_nothing_to_do(vs):
    x, q, targets, _ = make(5, 3, 8, torch.float32, 2, False, 6)
    lp, lse, ent, tv, ti = vs.vs_flat_logprob(x, q[:0], targets[:0], 2)
    assert lp.shape == (0, 2) and lse.shape == (0,) and tv.shape == (0, 2)
    lp, lse, ent, tv, ti = vs.vs_flat_logprob(x[:0], q, targets, 2)
    assert (lse == -INF).all() and (ent == 0).all() and (ti == -1).all() and (tv == -INF).all() and (lp == 0).all()
    dx, dq, db = vs.vs_flat_logprob_grad(x, q[:0], lse[:0])
    assert dq.shape == (0, 8) and (dx == 0).all() and (db == 0).all()
    dx, dq, db = vs.vs_flat_logprob_grad(x[:0], q, lse)
    assert dx.shape == (0, 8) and (dq == 0).all()


def test_nan_queries_answer_nan(vs):
    for nq in (4, 90):
        x, q, _, _ = make(300, nq, 64, torch.bfloat16, 0, False, 8)
        q[2, 5] = float("nan")
        lse = vs.vs_flat_logprob(x, q)[1]
        assert lse[2].isnan() and lse.isnan().sum() == 1


def check_grad(vs, x, q, targets, lse, ent, scale, bias, seed, entropy=True, g_lse=True):
    g = torch.Generator().manual_seed(seed)
    nq = q.shape[0]
    gl = None if targets is None else torch.randn(nq, targets.shape[1], generator=g).cuda()
    gz = torch.randn(nq, generator=g).cuda() if g_lse else None
    gh = torch.randn(nq, generator=g).cuda() if entropy else None
    dx, dq, db = vs.vs_flat_logprob_grad(x, q, lse, targets, gl, gz, ent, gh, scale, bias)
    torch.cuda.synchronize()
    (rq, rx, rb), (tq, tx, tb) = logprob_grad(x, q, targets, lse, ent, gl, gz, gh, scale, bias)
    close(dq, rq, tq, "dq")
    close(dx, rx, tx, "dx")
    close(db, rb, tb, "dbias")
    return dx, dq, db


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nb,nq,d", [(1, 1, 1), (5, 2, 3), (130, 1, 33), (128, 128, 64), (300, 129, 100), (2000, 40, 768),
                                     (65, 700, 31), (1, 200, 64), (20_000, 3, 40)])
@pytest.mark.parametrize("masked", [False, True])
def test_gradients(vs, dtype, nb, nq, d, masked):
    x, q, targets, bias = make(nb, nq, d, DTYPES[dtype], 3, masked and nb > 5, nb + d, grid=False)
    ref = logprob(x, q, targets, 0, 0.25, bias)
    lse, ent = ref["lse"].float().cuda(), ref["entropy"].float().cuda()
    check_grad(vs, x, q, targets, lse, ent, 0.25, bias, 2)


# what is tiled in larger tiles: pairs of long 16-bit rows; a gradient of many rows, stored as it is summed; one of few
# tiles whose sums are long
@pytest.mark.parametrize("dtype,nb,nq,d", [("bf16", 4100, 2100, 640), ("fp16", 4097, 2049, 700), ("bf16", 41_000, 130, 100),
                                           ("fp32", 41_003, 70, 33), ("fp32", 8200, 4000, 600)])
def test_large_gradients(vs, dtype, nb, nq, d):
    x, q, targets, bias = make(nb, nq, d, DTYPES[dtype], 2, True, nb + d, grid=False)
    ref = logprob(x, q, targets, 0, 0.1, bias)
    check_grad(vs, x, q, targets, ref["lse"].float().cuda(), ref["entropy"].float().cuda(), 0.1, bias, 2)


def test_gradients_in_chunks(vs):
    """More pairs than one piece of G holds: rows are taken in several chunks, queries' sums go on across them."""
    x, q, targets, bias = make(70_001, 1100, 24, torch.float32, 2, True, 9, grid=False)
    assert 70_001 * 1152 * 8 > 2 * (256 << 20)
    lse, ent = check_forward(vs, x, q, targets, 0, 0.25, bias)
    check_grad(vs, x, q, targets, lse, ent, 0.25, bias, 3)


def test_gradients_agree_with_differences(vs):
    """The loss along a direction, in 64 bits, against the gradient's component."""
    x, q, targets, _ = make(200, 9, 48, torch.float32, 2, False, 10, grid=False)
    targets = targets.clamp(0, 199)
    bias = torch.randn(200, device="cuda") * 0.3
    g = torch.Generator().manual_seed(1)
    gl, gz, gh = (torch.randn(9, 2, generator=g), torch.randn(9, generator=g), torch.randn(9, generator=g))
    _, lse, ent, _, _ = vs.vs_flat_logprob(x, q, targets, 0, 0.3, bias)
    dx, dq, db = vs.vs_flat_logprob_grad(x, q, lse, targets, gl.cuda(), gz.cuda(), ent, gh.cuda(), 0.3, bias)

    def loss(x, q, b):
        r = logprob(x, q, targets, 0, 0.3, b)
        return (gl.double() * r["logp"]).sum() + (gz.double() * r["lse"]).sum() + (gh.double() * r["entropy"]).sum()

    ux, uq, ub = (torch.randn(t.shape, generator=g, dtype=torch.float64) for t in (x, q, bias))
    e = 1e-4
    X, Q, B = x.double().cpu(), q.double().cpu(), bias.double().cpu()
    along = (loss(X + e * ux, Q + e * uq, B + e * ub) - loss(X - e * ux, Q - e * uq, B - e * ub)) / (2 * e)
    inner = (dx.double().cpu() * ux).sum() + (dq.double().cpu() * uq).sum() + (db.double().cpu() * ub).sum()
    size = (dx.double().cpu() * ux).abs().sum() + (dq.double().cpu() * uq).abs().sum() + (db.double().cpu() * ub).abs().sum()
    # third derivatives of order 1 along a direction of some 100 components: e^2 times their size stays below 1e-5 of it
    assert abs(along - inner) <= 1e-5 * size


def test_same_target_twice_and_padded_queries(vs):
    x, q, _, _ = make(200, 6, 64, torch.float32, 0, False, 11, grid=False)
    targets = torch.tensor([[3, 3], [5, -1], [-1, -1], [7, 8], [199, 0], [-7, 900]], device="cuda")
    q[2], q[5] = float("nan"), INF                      # padding: no labels, no gradient, anything inside
    _, lse, ent, _, _ = vs.vs_flat_logprob(x, q, targets)
    g = torch.ones(6, 2, device="cuda")
    dx, dq, db = vs.vs_flat_logprob_grad(x, q, lse, targets, g)
    live = torch.tensor([0, 1, 3, 4], device="cuda")
    (rq, rx, rb), (tq, tx, tb) = logprob_grad(x, q[live], targets[live], lse[live], None, g[live], None, None, 1.0, None)
    close(dq[live], rq, tq, "dq")
    close(dx, rx, tx, "dx")
    close(db, rb, tb, "dbias")
    assert (dq[2] == 0).all() and (dq[5] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nb,d", [(300, 100), (4100, 640)])
def test_padded_queries_among_many(vs, dtype, nb, d):
    """A batch whose last third is padding: targets of -1, no gradients, whatever it holds."""
    nq, live = 2100 if nb > 1000 else 90, 1400 if nb > 1000 else 60
    x, q, targets, _ = make(nb, nq, d, DTYPES[dtype], 1, False, 21, grid=False)
    q[live::2], q[live + 1::2] = float("nan"), INF
    targets[live:] = -1
    lse = vs.vs_flat_logprob(x, q, targets, scale=0.1)[1]
    g = torch.ones(nq, 1, device="cuda")
    dx, dq, db = vs.vs_flat_logprob_grad(x, q, lse, targets, g, scale=0.1)
    ref = logprob_grad(x, q[:live], targets[:live], lse[:live], None, g[:live], None, None, 0.1, None)
    for got, want, tol, what in zip((dq[:live], dx, db), *ref, ("dq", "dx", "dbias")):
        close(got, want, tol, what)
    assert (dq[live:] == 0).all()


def test_only_what_is_wanted(vs):
    x, q, targets, bias = make(400, 90, 64, torch.bfloat16, 1, True, 12)
    lse, ent = vs.vs_flat_logprob(x, q, targets, 0, 0.25, bias)[1:3]
    g = torch.ones(90, 1, device="cuda")
    whole = vs.vs_flat_logprob_grad(x, q, lse, targets, g, scale=0.25, bias=bias)
    for i in range(3):
        want = [j == i for j in range(3)]
        one = vs.vs_flat_logprob_grad(x, q, lse, targets, g, scale=0.25, bias=bias, want_dx=want[0], want_dq=want[1], want_dbias=want[2])
        assert torch.equal(one[i], whole[i]) and all(one[j] is None for j in range(3) if j != i)


@pytest.mark.parametrize("scale", [0.0, -0.25, 3.7])
@pytest.mark.parametrize("nq", [8, 100])
def test_scales(vs, scale, nq):
    x, q, targets, bias = make(900, nq, 50, torch.float32, 2, True, 13)
    ref = logprob(x, q, targets, 0, scale, bias)
    lse, ent, = vs.vs_flat_logprob(x, q, targets, 0, scale, bias)[1:3]
    t, th = logprob_tolerance(ref, x, q, scale, bias)
    close(lse, ref["lse"], t, "lse")
    close(ent, ref["entropy"], th, "entropy")
    check_grad(vs, x, q, targets, lse, ent, scale, bias, 4)


@pytest.mark.parametrize("size", [1e-30, 1e-4, 1e6, 1e18])
def test_magnitudes(vs, size):
    """fp32 components far from 1, of rows that differ in size: the 16-bit parts are relative to their row."""
    x, q, targets, _ = make(300, 80, 40, torch.float32, 2, False, 14, grid=False)
    x = x * size * (2.0 ** torch.arange(-6, 6, 12 / 300, device="cuda"))[:300, None].contiguous()
    q = q / size
    lse, ent = check_forward(vs, x, q, targets, 0, 0.25, None)
    check_grad(vs, x, q, targets, lse, ent, 0.25, None, 5)


def test_rows_beyond_32_bit_offsets(vs):
    """2.4e9 components: the last rows are found, and their scores are those of a small call."""
    nb, d = 3_100_000, 768
    x = torch.zeros(nb, d, dtype=torch.float16, device="cuda")
    q = (torch.randn(66, d, generator=torch.Generator().manual_seed(3)) * 0.1).half().cuda()
    x[nb - 3:] = q[:3] * 8
    targets = torch.full((66, 1), nb - 2, device="cuda")
    for n in (2, 66):
        lp, lse, _, tv, ti = vs.vs_flat_logprob(x, q[:n].contiguous(), targets[:n].contiguous(), 2)
        own = (q[:n].double() @ x[nb - 3:].double().t())
        want = torch.logsumexp(torch.cat((own, torch.full((n, 1), float(np.log(nb - 3)), device="cuda", dtype=torch.float64)), 1), 1)
        assert (lse.double() - want).abs().max() < 1e-4
        assert (ti[0, 0], ti[1, 0]) == (nb - 3, nb - 2)
        assert (lp[:, 0].double() - (own[:, 1] - want)).abs().max() < 1e-4
    lse = vs.vs_flat_logprob(x, q, None)[1]
    dx, dq, db = vs.vs_flat_logprob_grad(x, q, lse, targets, -torch.ones(66, 1, device="cuda"))
    p = torch.exp((q.double() @ x[nb - 2].double()) - lse.double())
    assert (db[nb - 2].double() - (p - 1).sum()).abs() < 1e-4 * 66
    assert (dx[nb - 2].double() - ((p - 1)[:, None] * q.double()).sum(0)).abs().max() < 2e-2


def test_equal_calls_give_equal_bits_on_any_stream(vs):
    x, q, targets, bias = make(5000, 300, 96, torch.float32, 2, True, 15, grid=False)
    g = torch.randn(300, 2, device="cuda")
    a = vs.vs_flat_logprob(x, q, targets, 5, 0.25, bias)
    da = vs.vs_flat_logprob_grad(x, q, a[1], targets, g, scale=0.25, bias=bias)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for st in streams:                                   # two calls at once
        with torch.cuda.stream(st):
            b = vs.vs_flat_logprob(x, q, targets, 5, 0.25, bias)
            outs.append(b + vs.vs_flat_logprob_grad(x, q, b[1], targets, g, scale=0.25, bias=bias))
    torch.cuda.synchronize()
    for o in outs:
        for u, v in zip(a + da, o):
            assert torch.equal(u, v)


@pytest.mark.parametrize("nq,dtype", [(3, "bf16"), (200, "bf16"), (200, "fp32")])
def test_captured_and_replayed(vs, nq, dtype):
    x, q, targets, bias = make(3000, nq, 96, DTYPES[dtype], 1, True, 16, grid=False)
    g = torch.randn(nq, 1, device="cuda")

    def both():
        f = vs.vs_flat_logprob(x, q, targets, 4, 0.25, bias)
        return f + vs.vs_flat_logprob_grad(x, q, f[1], targets, g, scale=0.25, bias=bias)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for r in range(4):
        q.copy_((torch.randn(q.shape, generator=torch.Generator().manual_seed(r)) * 0.5).to(q.dtype))
        want = [t.clone() for t in both()]               # eager work between replays
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(out, want):
            assert torch.equal(u, v)


def test_binding_refuses_shapes_and_types(vs):
    x, q, targets, bias = make(50, 4, 8, torch.float32, 1, True, 17)
    with pytest.raises(ValueError):
        vs.vs_flat_logprob(x, q[:, :7].contiguous())
    with pytest.raises(ValueError):
        vs.vs_flat_logprob(x.t(), q)
    with pytest.raises(TypeError):
        vs.vs_flat_logprob(x, q.half())
    with pytest.raises(TypeError):
        vs.vs_flat_logprob(x.double(), q.double())
    with pytest.raises(TypeError):
        vs.vs_flat_logprob(x, q, targets.int())
    with pytest.raises(ValueError):
        vs.vs_flat_logprob(x, q, targets[:3])
    with pytest.raises(ValueError):
        vs.vs_flat_logprob(x, q, bias=bias[:49].contiguous())
    with pytest.raises(vs.VSError):
        vs.vs_flat_logprob(x, q, k=65)
    lse = vs.vs_flat_logprob(x, q)[1]
    with pytest.raises(TypeError):
        vs.vs_flat_logprob_grad(x, q, None)
    with pytest.raises(ValueError):
        vs.vs_flat_logprob_grad(x, q, lse, targets, torch.ones(4, 2, device="cuda"))
    with pytest.raises(vs.VSError):
        vs.vs_flat_logprob_grad(x, q, lse, g_entropy=lse)
    # rows that start in the middle of a 16-byte piece are copied first
    flat = torch.zeros(51 * 8 + 1, device="cuda")
    odd = flat[1:1 + 50 * 8].view(50, 8)
    odd.copy_(x)
    assert torch.equal(vs.vs_flat_logprob(odd, q, bias=bias)[1], vs.vs_flat_logprob(x, q, bias=bias)[1])

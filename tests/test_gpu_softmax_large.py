"""Calls whose launches would exceed 2^32 threads in one dimension go in pieces or in two dimensions (GPU)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
MANY = (1 << 24) + 5                               # queries: a workgroup of 256 threads each is 2^32 threads


@pytest.fixture(scope="module")
def vs():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2401_08281_amd as vs
    vs.softmax_lib()
    yield vs
    torch.cuda.empty_cache()


def test_log_probabilities_of_2_24_queries(vs):
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(MANY, 1, device="cuda", generator=g).half()
    x = torch.randn(3, 1, device="cuda", generator=g).half()
    lse, ent = vs.vs_flat_logprob(x, q)[1:3]
    for a in (0, MANY - 70_000):
        s = q[a:a + 70_000].double() @ x.double().t()
        want = torch.logsumexp(s, 1)
        p = torch.exp(s - want[:, None])
        assert (lse[a:a + 70_000].double() - want).abs().max() < 1e-5
        assert (ent[a:a + 70_000].double() + (p * (s - want[:, None])).sum(1)).abs().max() < 1e-5
    lse, ent = vs.vs_flat_logprob(x[:0], q)[1:3]
    assert (lse == -float("inf")).all() and (ent == 0).all()


def test_log_probabilities_over_2_28_rows(vs):
    """Prepared copies take sixteen threads a row."""
    g = torch.Generator(device="cuda").manual_seed(2)
    nb = (1 << 28) + 77
    x = torch.randn(nb, 1, device="cuda", generator=g, dtype=torch.float16)
    q = torch.randn(65, 1, device="cuda", generator=g).half()
    x[nb - 3] = 30.0
    q[7] = 2.0
    targets = torch.full((65, 1), nb - 3, device="cuda")
    lp, lse, _, tv, ti = vs.vs_flat_logprob(x, q, targets, 1)
    for i in (0, 7, 64):
        s = q[i].double() * x[:, 0].double()
        want = torch.logsumexp(s, 0)
        assert (lse[i].double() - want).abs() < 1e-3
        assert (lp[i, 0].double() - (s[nb - 3] - want)).abs() < 1e-3
    assert ti[7, 0] == nb - 3
    few = vs.vs_flat_logprob(x, q[:3].contiguous(), None, 1)
    assert (few[1] - lse[:3]).abs().max() < 1e-3


def test_gradients_of_2_32_components(vs):
    nq, nb, d = 65_600, 3, 65_536
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.empty(nq, d, dtype=torch.bfloat16, device="cuda")
    for a in range(0, nq, 4100):
        q[a:a + 4100] = torch.randn(4100, d, device="cuda", generator=g).bfloat16()
    x = torch.randn(nb, d, device="cuda", generator=g).bfloat16()
    targets = torch.randint(0, nb, (nq, 1), device="cuda", generator=g)
    scale = 0.004
    logp, lse = vs.vs_flat_logprob(x, q, targets, scale=scale)[:2]
    gl = -torch.ones(nq, 1, device="cuda")
    dx, dq, db = vs.vs_flat_logprob_grad(x, q, lse, targets, gl, scale=scale)
    G = []
    for a in range(0, nq, 4100):
        s = scale * (q[a:a + 4100].float() @ x.float().t()).double()
        p = torch.softmax(s, 1)
        G.append(p - torch.nn.functional.one_hot(targets[a:a + 4100, 0], nb))
    G = torch.cat(G)
    assert (db.double() - G.sum(0)).abs().max() < 1e-3 * G.abs().sum(0).max()
    for rows in (slice(0, 100), slice(nq - 100, nq)):
        want = scale * (G[rows] @ x.double())
        assert (dq[rows].double() - want).abs().max() <= 2.0 ** -7 * want.abs().max()
    cols = torch.tensor([0, 1, 255, 32_767, 65_535], device="cuda")
    want = scale * (G.t() @ q[:, cols].double())
    assert (dx[:, cols].double() - want).abs().max() <= 2.0 ** -7 * want.abs().max()


def test_attention_of_2_24_queries(vs):
    g = torch.Generator(device="cuda").manual_seed(4)
    t = lambda *s: torch.randn(*s, device="cuda", generator=g)
    ix = vs.IVFPQ(2, vs.METRIC_IP, t(2, 2), t(2, 16, 1), 4)
    ix.add(t(5, 2))
    q = t(MANY, 2)
    go = t(MANY, 2)
    # halves of the batch in two calls: the same queries side by side, so the same bits
    cut = MANY // 2 // 64 * 64
    for nprobe in (0, 1):
        out, lse = ix.attend(q, nprobe, 0.5)
        dq = ix.attend_grad(q, nprobe, 0.5, lse, go)
        for part in (slice(0, cut), slice(cut, MANY)):
            o, z = ix.attend(q[part].contiguous(), nprobe, 0.5)
            assert torch.equal(out[part], o) and torch.equal(lse[part], z)
            assert torch.equal(dq[part], ix.attend_grad(q[part].contiguous(), nprobe, 0.5, z, go[part].contiguous()))
        assert lse.isfinite().all()

"""How far the parts that operands are held in may be off where components differ in size (GPU)."""
import pytest
import torch

from softmax_reference import HALF, U, f64, logprob_grad
from test_gpu_logprob import DTYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vs():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2401_08281_amd as vs
    vs.softmax_lib()
    return vs


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [10, 20, 26])
@pytest.mark.parametrize("nb,nq,d", [(300, 40, 64), (300, 200, 100), (20_000, 150, 100), (6000, 2100, 640)])
def test_a_large_row_leaves_the_others_their_bits(vs, nb, nq, d, bits, dtype):
    """One row 2^bits larger than the others, with next to no probability: columns are held relative to their largest
    component, brought to 2^14 at least, in parts whose smallest half step is 2^-25: 2^-39 of the largest (and 2^-24 of
    themselves in two parts; 16-bit values are exact above that)."""
    g = torch.Generator().manual_seed(bits + nb)
    x = torch.randn(nb, d, generator=g) * 0.5
    x[nb // 2] *= 2.0 ** bits
    q = torch.randn(nq, d, generator=g) * 0.5
    x, q = x.to(DTYPES[dtype]).cuda(), q.to(DTYPES[dtype]).cuda()
    bias = torch.zeros(nb, device="cuda")
    bias[nb // 2] = -2.0 ** (bits + 8)
    targets = torch.randint(0, nb // 2, (nq, 1), generator=g).cuda()
    lse = vs.vs_flat_logprob(x, q, None, 0, 0.25, bias)[1]
    # (rows without the large one, of which nothing is left in any sum)
    keep = torch.arange(nb, device="cuda") != nb // 2
    gl = -torch.ones(nq, 1, device="cuda")
    dx, dq, db = vs.vs_flat_logprob_grad(x, q, lse, targets, gl, scale=0.25, bias=bias)
    (rq, _, _), (tq, _, _) = logprob_grad(x[keep], q, targets, lse, None, gl, None, None, 0.25, bias[keep])
    s = 0.25 * f64(q) @ f64(x[keep]).t() - f64(lse)[:, None]
    G = torch.exp(s).scatter_add(1, targets.cpu(), -torch.ones(nq, 1, dtype=torch.float64))
    top = f64(x).abs().amax(0)
    tol = tq + 0.25 * 2.0 ** -39 * G.abs().sum(1, keepdim=True) * top
    worst = ((f64(dq) - rq).abs() / tol).max()
    assert worst <= 1, float(worst)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [10, 20, 26])
@pytest.mark.parametrize("nb,nq,d", [(300, 40, 64), (3000, 200, 100), (41_000, 130, 100)])
def test_a_small_weight_leaves_a_row_its_gradient(vs, nb, nq, d, bits, dtype):
    """One query whose loss weighs 2^-bits of the others', alone in asking for a row that the others all but exclude."""
    g = torch.Generator().manual_seed(bits + nb)
    x = torch.randn(nb, d, generator=g) * 0.25
    q = torch.randn(nq, d, generator=g) * 0.25
    i, j = nq // 3, nb - 5
    q[:, 0], x[:, 0] = 4.0, 0.0
    q[i, 0], x[j, 0] = -4.0, -64.0                  # <q, x_j> about -256 for all but query i, +256 for it
    x, q = x.to(DTYPES[dtype]).cuda(), q.to(DTYPES[dtype]).cuda()
    targets = torch.randint(0, nb - 100, (nq, 1), generator=g).cuda()
    lse = vs.vs_flat_logprob(x, q)[1]
    gl = -torch.ones(nq, 1, device="cuda")
    gl[i] = -2.0 ** -bits
    dx, dq, db = vs.vs_flat_logprob_grad(x, q, lse, targets, gl)
    s = f64(q) @ f64(x).t()
    p = torch.softmax(s, 1)
    G = -f64(gl) * p
    G.scatter_add_(1, targets.cpu(), f64(gl))
    want = G[:, j] @ f64(q)                         # 2^-bits q_i, up to e^-256
    # p is 1 up to the scores' and the normaliser's roundings (sizes of 256, some d of them); G has 11 bits in one part and 22
    # in two; columns of (bound q) keep 2^-39 of their largest, 4 |q_t| for the others' bound of 4, and |G| is at most half of
    # query i's bound
    part = HALF[torch.float16] if dtype == "bf16" else 2.0 ** -20
    rel = 2 * (d + 40) * U * 256 + 2.0 ** -19 * 256 + part + HALF[DTYPES[dtype]]
    tol = rel * want.abs() + 2.0 ** -39 * 0.5 * 4.0 * f64(q).abs().amax(0) + 1e-30
    worst = ((f64(dx[j]) - want).abs() / tol).max()
    assert worst <= 1, float(worst)

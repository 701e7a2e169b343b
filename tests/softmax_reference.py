"""The softmax operators in 64 bits on the CPU, and how far 32-bit results may be off (worked out from
the number of roundings, not from results)."""
import torch

U = 2.0 ** -24                                       # half a step of fp32, relative
HALF = {torch.float32: U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
INF = float("inf")


def f64(t):
    return None if t is None else t.detach().double().cpu()


def scores(x, q, scale, bias):
    s = scale * (f64(q) @ torch.nan_to_num(f64(x), 0.0, 0.0, 0.0).t())
    if bias is None:
        return s
    return torch.where(f64(bias) == -INF, torch.tensor(-INF, dtype=torch.float64), s + f64(bias))


def softmax(s):
    """(lse, p, logp) of rows that may hold nothing but -inf."""
    lse = torch.logsumexp(s, 1) if s.shape[1] else torch.full((s.shape[0],), -INF, dtype=torch.float64)
    base = torch.where(lse == -INF, torch.zeros_like(lse), lse)[:, None]
    logp = s - base
    return lse, torch.exp(logp), logp


def score_error(x, q, scale, bias):
    """A score: d products of 16-bit numbers are exact, their fp32 sum in any order loses d roundings of the sum of their
    sizes; scaling, bias and the subtraction of the maximum three more.  fp32 vectors go as two fp16 parts whose
    product of tails (2^-22 of |q||x|) is left out and whose tails are rounded (2^-22 each): 2^-21 |q||x|, twice over
    where a sum of components stands for the norm."""
    x, q = torch.nan_to_num(f64(x), 0.0, 0.0, 0.0), f64(q)
    size = abs(scale) * (q.abs() @ x.abs().t()).amax() + (0.0 if bias is None else f64(bias)[f64(bias).isfinite()].abs().amax())
    e = (x.shape[1] + 8) * U * size
    split = abs(scale) * 2.0 ** -20 * q.norm(dim=1).amax() * x.norm(dim=1).amax()
    return float(e + split)


def logprob(x, q, targets, k, scale, bias):
    s = scores(x, q, scale, bias)
    lse, p, logp = softmax(s)
    ent = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    out = {"lse": lse, "entropy": ent}
    if targets is not None:
        t = targets.cpu()
        ok = (t >= 0) & (t < x.shape[0])
        lp = torch.gather(logp, 1, t.clamp(0, max(x.shape[0] - 1, 0))) if x.shape[0] else torch.zeros(t.shape, dtype=torch.float64)
        out["logp"] = torch.where(ok, lp, torch.zeros_like(lp))
    if k:
        n = min(k, x.shape[0])
        v, i = torch.sort(logp, dim=1, descending=True, stable=True)
        top = torch.full((q.shape[0], k), -INF, dtype=torch.float64)
        ids = torch.full((q.shape[0], k), -1, dtype=torch.int64)
        top[:, :n] = v[:, :n]
        ids[:, :n] = torch.where(v[:, :n] > -INF, i[:, :n], torch.full_like(i[:, :n], -1))
        out["top_logp"], out["top_ids"] = top, ids
    return out


def logprob_tolerance(ref, x, q, scale, bias):
    """lse: the scores' error, the sums' (some 300 additions and an exponential each, relative to the sum) and its own
    rounding.  Entropy -sum p logp: its derivative for a score is p (logp + H), in sum at most 2 H."""
    es = score_error(x, q, scale, bias) if x.shape[0] else 0.0
    lse = ref["lse"]
    big = lse[lse.isfinite()].abs().amax() if lse.isfinite().any() else 0.0
    t = es + 512 * U + 4 * U * big
    h = ref["entropy"].amax() + 1.0
    return float(t), float(2 * h * t + 1024 * U * h)


def logprob_grad(x, q, targets, lse, ent, g_logp, g_lse, g_entropy, scale, bias):
    """Gradients, and a bound of the error of each of their elements."""
    dt = x.dtype
    xd, qd, s = torch.nan_to_num(f64(x), 0.0, 0.0, 0.0), f64(q), scores(x, q, scale, bias)
    nq, nb = s.shape
    z = f64(lse)
    logp = s - torch.where(z == -INF, torch.zeros_like(z), z)[:, None]
    p = torch.exp(logp)
    gl = torch.zeros(nq, 0, dtype=torch.float64) if g_logp is None else f64(g_logp)
    t = torch.zeros(nq, 0, dtype=torch.int64) if g_logp is None else targets.cpu()
    ok = (t >= 0) & (t < nb)
    gl = torch.where(ok, gl, torch.zeros_like(gl))
    c = -gl.sum(1) + (0.0 if g_lse is None else f64(g_lse))
    ge = torch.zeros(nq, dtype=torch.float64) if g_entropy is None else f64(g_entropy)
    h = torch.zeros(nq, dtype=torch.float64) if g_entropy is None else f64(ent)
    inner = torch.where(p > 0, logp + h[:, None], torch.zeros_like(p))
    soft = p * c[:, None] - ge[:, None] * p * inner
    G = soft.clone().scatter_add_(1, t.clamp(0, nb - 1), gl)
    exists = s > -INF
    G = torch.where(exists, G, torch.zeros_like(G))
    dq, dx, db = scale * (G @ xd), scale * (G.t() @ qd), G.sum(0)
    # p is off by the scores' error and that of the given lse; G by that, some roundings, and its 16-bit parts
    es = score_error(x, q, scale, bias) + 8 * U * float(z[z.isfinite()].abs().amax() if z.isfinite().any() else 0.0) + 8 * U
    size = p * (c.abs()[:, None] + ge.abs()[:, None] * (inner.abs() + 1.0))
    eg = torch.where(exists, 2 * es * size + 8 * U * (size + G.abs()), torch.zeros_like(G))
    bound = 2.0 * (c.abs() + gl.abs().sum(1) + ge.abs() * (0.37 + h.abs()))      # a power of two above the sum
    parts = 2.0 ** -21 if dt == torch.float32 else HALF[torch.float16]           # G in one or two fp16 parts
    eh = eg + parts * G.abs() + torch.where(exists, 2.0 ** -38 * bound[:, None], torch.zeros_like(G))
    # (the other operand's parts: 2^-21 in two, exact in one but for what lies 2^-22 below its column's largest)
    other = 2.0 ** -21
    def product(e, g, v, n):
        return abs(scale) * (e @ v.abs() + (other + (n + 8) * U) * (g.abs() @ v.abs())
                             + 2.0 ** -32 * g.abs().sum(1, keepdim=True) * v.abs().amax(0, keepdim=True))
    tq = product(eh, G, xd, nb) + HALF[dt] * dq.abs() + 1e-30
    tx = product(eh.t(), G.t(), qd, nq) + 2.0 ** -38 * abs(scale) * (bound[:, None] * qd.abs()).amax(0) * nq \
        + HALF[dt] * dx.abs() + 1e-30
    tb = eg.sum(0) + (nq + 8) * U * G.abs().sum(0) + 1e-30
    if dt == torch.float16:                         # results below the smallest normal number are rounded to its steps
        tq, tx = tq + 2.0 ** -25, tx + 2.0 ** -25
    return (dq, dx, db), (tq, tx, tb)


def decode(centroids, codebooks, codes, list_of):
    M, K, dsub = codebooks.shape
    c = torch.stack((codes & 15, codes >> 4), dim=2).reshape(codes.shape[0], M).long()
    words = codebooks.reshape(M * K, dsub)[c + torch.arange(M) * K].reshape(codes.shape[0], M * dsub)
    return centroids[list_of] + words


def attend(rows, q, sees, dk, v0, scale):
    """rows [n, d] fp64; sees [nq, n]: which rows take part.  (out, lse, p)."""
    s = scale * (f64(q) @ rows[:, :dk].t())
    s = torch.where(sees, s, torch.full_like(s, -INF))
    lse, p, _ = softmax(s)
    return p @ rows[:, v0:], lse, p


def attend_tolerance(rows, q, p, dk, v0, scale, M, dtype, out):
    """A score: dk products and M + 8 additions, relative to the sum of sizes.  out: twice the scores' error (weights and
    normaliser), the additions of n weights, and for 16-bit queries a 16-bit rounding of weights and values each."""
    n = rows.shape[0]
    es = (dk + M + 8) * U * abs(scale) * float((f64(q).abs() @ rows[:, :dk].abs().t()).amax()) * 3 \
        + 2.0 ** -20 * abs(scale) * float(f64(q).norm(dim=1).amax() * rows[:, :dk].norm(dim=1).amax())
    spread = p @ rows[:, v0:].abs()
    low = 0.0 if dtype == torch.float32 else 2 * HALF[torch.float16]
    return es, (2 * es + (n + 64) * U + 2.0 ** -20 + low) * (spread + rows[:, v0:].abs().amax(0) * 2.0 ** -11) \
        + HALF[dtype] * out.abs() + 2.0 ** -25


def attend_grad(rows, q, p, g_out, g_lse, dk, v0, scale, M, es):
    """(dq, bound of its elements' error): the two sums sum p dp k and (sum p dp) (sum p k) are formed apart, so their
    sizes count, not their difference."""
    dt = q.dtype
    k, v, g = rows[:, :dk], rows[:, v0:], f64(g_out)
    dp = g @ v.t()
    mean = (p * dp).sum(1, keepdim=True)
    gl = torch.zeros(q.shape[0], 1, dtype=torch.float64) if g_lse is None else f64(g_lse)[:, None]
    dq = scale * ((p * (dp - mean + gl)) @ k)
    dpa = g.abs() @ v.abs().t()
    big = (p * dpa) @ k.abs() + ((p * dpa).sum(1, keepdim=True) + gl.abs()) * (p @ k.abs())
    low = 0.0 if dt == torch.float32 else 4 * HALF[torch.float16]
    tol = abs(scale) * (4 * es + (rows.shape[0] + dk + M + 64) * U + 2.0 ** -19 + low) * big + HALF[dt] * dq.abs() + 2.0 ** -25
    return dq, tol

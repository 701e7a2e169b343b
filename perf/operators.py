"""Softmax over the rows of an index: the operators, their plain forms and the work to time.

Where a search returns the k best rows, these weigh all of them:
  logprob       log-probabilities of given rows under the softmax of exact inner products, with the
                entropy and the k best alternatives (retrieval heads, softmax layers over an item table)
  logprob_grad  its gradients for the queries, the rows and the bias
  attend        attention over the vectors of a 4-bit IVF-PQ index (all lists, or the probed ones)
  attend_grad   its gradient for the queries; the index stays as it is

`run` is one call.  With `own` false it computes the definition with elementary torch operations,
with `own` true it calls the library.  Scores that decide an order (alternatives, probed lists) come
from values on a binary grid, as 8-bit embeddings have them: their fp32 sums are exact in any order.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
PLAIN_ELEMENTS = 1 << 28          # scores the plain forms hold at a time
INF = float("inf")


# ---- cases ---------------------------------------------------------------------------------------

def listed():
    return [
        # one hidden state against a table of 100,003 embeddings: latency, one read of the table
        dict(name="logprob_one", op="logprob", nq=1, nb=100_003, d=768, dtype="bf16", nt=1, k=10, bias="none"),
        # an evaluation batch of embeddings against a 64k table, top 5
        dict(name="logprob_batch", op="logprob", nq=4096, nb=65_536, d=768, dtype="bf16", nt=1, k=5, bias="none"),
        # item scores with popularity corrections and deleted items, several positives per query, ragged
        dict(name="logprob_items", op="logprob", nq=1000, nb=200_003, d=100, dtype="fp32", nt=3, k=10, bias="masked"),
        # contrastive training inside one batch
        dict(name="grad_in_batch", op="logprob_grad", nq=1024, nb=1024, d=96, dtype="fp32", nt=1, bias="none",
             entropy=False),
        # training against a whole table of embeddings
        dict(name="grad_table", op="logprob_grad", nq=4096, nb=65_536, d=768, dtype="bf16", nt=1, bias="none",
             entropy=False),
        # an entropy-regularised loss with a trained bias, ragged sizes, half precision
        dict(name="grad_entropy", op="logprob_grad", nq=777, nb=30_011, d=100, dtype="fp16", nt=2, bias="masked",
             entropy=True),
        # one small step over a short memory: launches and latency
        dict(name="attend_one", op="attend", nq=1, nb=4097, d=96, M=32, nlist=16, nprobe=0, dk=96, v0=0, dtype="fp16",
             limits=False),
        # one decoding step: the query heads that share a key-value memory of 131,072 positions
        dict(name="attend_step", op="attend", nq=8, nb=131_072, d=256, M=64, nlist=1, nprobe=0, dk=128, v0=128,
             dtype="bf16", limits=False),
        # a prompt over the same kind of memory, every query up to its own position
        dict(name="attend_prompt", op="attend", nq=2048, nb=16_384, d=256, M=64, nlist=1, nprobe=0, dk=128, v0=128,
             dtype="bf16", limits=True),
        # retrieval attention: each query reads its 32 nearest lists of a million 768-d vectors
        dict(name="attend_probe", op="attend", nq=1000, nb=1_000_000, d=768, M=64, nlist=4096, nprobe=32, dk=768, v0=0,
             dtype="fp32", limits=False),
        # the prompt's backward pass
        dict(name="attend_grad_prompt", op="attend_grad", nq=1024, nb=16_384, d=256, M=64, nlist=1, nprobe=0, dk=128,
             v0=128, dtype="bf16", limits=True),
        # fine-tuning of queries against a probed memory
        dict(name="attend_grad_probe", op="attend_grad", nq=333, nb=200_003, d=96, M=32, nlist=1000, nprobe=16, dk=96,
             v0=0, dtype="fp32", limits=False),
    ]


def _spread(rng, lo, hi):
    """An integer from lo to hi, even over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# (d, M, dk, v0) of 4-bit indexes: keys that are values, keys beside values, values that are a part of the keys
PQ_SHAPES = ((96, 32, 96, 0), (128, 32, 128, 0), (768, 64, 768, 0), (256, 64, 128, 128), (100, 20, 100, 0),
             (64, 32, 64, 0), (144, 36, 144, 16), (128, 64, 64, 64))


def draw(rng):
    op = rng.choice(("logprob", "logprob", "logprob_grad", "attend", "attend", "attend_grad"))
    dtype = rng.choice(("fp32", "fp16", "bf16"))
    if op.startswith("logprob"):
        d = rng.choice((32, 96, 100, 128, 768, rng.randint(8, 800)))
        nb = _spread(rng, 100, 300_000)
        nq = _spread(rng, 1, 8192)
        most = 4096 * 65_536 * 768 // (8 if dtype == "fp32" else 1)
        while nq > 1 and nq * nb * d > most:
            nq = (nq + 1) // 2
        case = dict(op=op, nq=nq, nb=nb, d=d, dtype=dtype, nt=rng.randint(1, 4), bias=rng.choice(("none", "masked")))
        if op == "logprob":
            case["k"] = rng.choice((0, 1, 5, rng.randint(1, 40)))
        else:
            case["entropy"] = rng.random() < 0.5
        return case
    d, M, dk, v0 = rng.choice(PQ_SHAPES)
    probed = rng.random() < 0.5
    nb = _spread(rng, 500, 300_000)
    nlist = max(2, int(math.sqrt(nb) * rng.uniform(0.5, 4.0))) if probed else rng.choice((1, 1, 7, 64))
    nprobe = min(_spread(rng, 1, 64), nlist) if probed else 0
    nq = _spread(rng, 1, 2048)
    visited = nb * nprobe // nlist + 1 if probed else nb
    while nq > 1 and nq * visited * M > 2048 * 16_384 * 64:
        nq = (nq + 1) // 2
    return dict(op=op, nq=nq, nb=nb, d=d, M=M, nlist=nlist, nprobe=nprobe, dk=dk, v0=v0, dtype=dtype,
                limits=rng.random() < 0.4)


# ---- inputs --------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _embeddings(g, n, d):
    """Embeddings on the grid of their 8-bit form: multiples of 1/64 up to 127/64."""
    return (_randn(g, n, d) * 32.0).round().clamp(-127, 127) / 64.0


def _scale(d):
    """A power of two near the inverse of the standard deviation of a score, times two."""
    return 2.0 ** round(math.log2(2.0 / (0.25 * math.sqrt(d))))


def _logprob_inputs(case, seed):
    g = _gen(seed)
    nq, nb, d, nt = case["nq"], case["nb"], case["d"], case["nt"]
    dt = DTYPES[case["dtype"]]
    x = _embeddings(g, nb, d)
    targets = torch.randint(0, nb, (nq, nt), generator=g, device="cuda")
    # a query resembles the row it should find
    q = x[targets[:, 0]] * 0.25 + _randn(g, nq, d) * 0.5
    q = (q * 64.0).round().clamp(-127, 127) / 64.0
    if case["op"] == "logprob_grad":        # no order to decide: values between the grid's
        x = x + _randn(g, nb, d) * 2.0 ** -9
        q = q + _randn(g, nq, d) * 2.0 ** -9
    bias = None
    if case["bias"] == "masked":
        bias = (_randn(g, nb) * 32.0).round() / 64.0
        bias[torch.rand(nb, generator=g, device="cuda") < 0.05] = -INF
    # every eighth query or so has no label in its last place
    drop = torch.rand(nq, generator=g, device="cuda") < 0.125
    targets[drop, nt - 1] = -1
    state = dict(case=case, x=x.to(dt), q=q.to(dt), bias=bias, targets=targets, scale=_scale(d))
    if case["op"] == "logprob_grad":
        state["g_logp"] = -(torch.rand(nq, nt, generator=g, device="cuda") + 0.5) / nq
        state["g_entropy"] = _randn(g, nq) * (0.1 / nq) if case["entropy"] else None
    return state


def _step(case):
    return max(1, PLAIN_ELEMENTS // max(case["nb"], 1))


def _unpack(codes):
    """[n, M / 2] bytes -> [n, M] code numbers."""
    return torch.stack((codes & 15, codes >> 4), dim=2).reshape(codes.shape[0], -1).long()


def _decode(centroids, codebooks, codes, list_of):
    """The vectors that codes stand for: centroid + concatenated codewords, fp32."""
    M, _, dsub = codebooks.shape
    c = _unpack(codes)
    words = codebooks.reshape(M * 16, dsub)[c + torch.arange(M, device=c.device) * 16]
    return centroids[list_of] + words.reshape(codes.shape[0], M * dsub)


def _attend_inputs(case, seed):
    g = _gen(seed)
    nq, nb, d, M, nlist, dk = case["nq"], case["nb"], case["d"], case["M"], case["nlist"], case["dk"]
    dt = DTYPES[case["dtype"]]
    centroids = (_randn(g, nlist, d) * 8.0).round() / 8.0
    codebooks = _randn(g, M, 16, d // M) * 0.5
    weight = torch.rand(nlist, generator=g, device="cuda") + 0.5
    list_of = torch.multinomial(weight, nb, replacement=True, generator=g).sort().values if nlist > 1 else \
        torch.zeros(nb, dtype=torch.int64, device="cuda")
    codes = torch.randint(0, 256, (nb, M // 2), generator=g, device="cuda", dtype=torch.uint8)
    pick = torch.randint(0, nb, (nq,), generator=g, device="cuda")
    near = _decode(centroids, codebooks, codes[pick], list_of[pick])[:, :dk]
    q = ((near * 0.75 + _randn(g, nq, dk)) * 16.0).round().clamp(-127, 127) / 16.0
    state = dict(case=case, q=q.to(dt), scale=1.0 / math.sqrt(dk), centroids=centroids, codebooks=codebooks,
                 codes=codes, list_of=list_of, limits=None)
    if case["limits"]:
        # query i of n stands at position (i + 1) nb / n; one in sixteen sees nothing yet
        lim = (torch.arange(1, nq + 1, device="cuda") * nb) // nq
        lim[torch.rand(nq, generator=g, device="cuda") < 1.0 / 16] = 0
        state["limits"] = lim
    if case["op"] == "attend_grad":
        state["g_out"] = _randn(g, nq, d - case["v0"]).to(dt)
    return state


def prepare(case, seed):
    if case["op"].startswith("logprob"):
        state = _logprob_inputs(case, seed)
        if case["op"] == "logprob_grad":    # the forward pass has returned these
            state["lse"], state["entropy"] = _normalisers(state)
        return state
    state = _attend_inputs(case, seed)
    if case["op"] == "attend_grad":
        state["lse"] = _attend_lse(state)
    if own:
        import paper_2401_08281_amd as vs
        ix = vs.IVFPQ(case["d"], vs.METRIC_IP, state["centroids"], state["codebooks"], 4)
        ix.set_coarse_metric(vs.METRIC_L2)
        ids = torch.arange(case["nb"], device="cuda")
        for a in range(0, case["nb"], 1 << 19):
            b = min(a + (1 << 19), case["nb"])
            ix.add(_decode(state["centroids"], state["codebooks"], state["codes"][a:b], state["list_of"][a:b]), ids[a:b])
        state["index"] = ix
    return state


# ---- plain forms ---------------------------------------------------------------------------------

def _scores(q, x, scale, bias):
    s = (q @ x.t()) * scale
    return s if bias is None else s + bias


def _normalisers(state):
    q, x, bias = state["q"].double(), state["x"].double(), state["bias"]
    lse, ent = [], []
    for a in range(0, q.shape[0], _step(state["case"]) // 2 + 1):
        s = _scores(q[a:a + _step(state["case"]) // 2 + 1], x, state["scale"], None if bias is None else bias.double())
        z = torch.logsumexp(s, 1)
        p = torch.exp(s - z[:, None])
        lse.append(z)
        ent.append(z - torch.where(p > 0, p * s, torch.zeros_like(s)).sum(1))
    return torch.cat(lse).float(), torch.cat(ent).float()


def _best(s, k):
    """Positions of the k largest values of every row, ties to the smaller position, -1 for values of -inf."""
    u = s.view(torch.int32)
    order = torch.where(u < 0, u ^ 0x7fffffff, u).long()       # as the values are ordered (-0 counts below 0)
    order = torch.where(s == 0, torch.zeros_like(order), order)
    key = (order << 32) | (s.shape[1] - 1 - torch.arange(s.shape[1], device=s.device))
    top = torch.topk(key, min(k, s.shape[1]), dim=1).values
    pos = s.shape[1] - 1 - (top & 0xffffffff)
    val = torch.gather(s, 1, pos)
    return val, torch.where(val == -INF, torch.full_like(pos, -1), pos)


def _plain_logprob(state):
    case = state["case"]
    q, x, bias, targets, k = state["q"].float(), state["x"].float(), state["bias"], state["targets"], case["k"]
    logp, lse, ent, tv, ti = [], [], [], [], []
    for a in range(0, q.shape[0], _step(case)):
        s = _scores(q[a:a + _step(case)], x, state["scale"], bias)
        t = targets[a:a + _step(case)]
        m = s.amax(1, keepdim=True)
        e = torch.exp(s - m)
        z = e.sum(1)
        lse.append(m[:, 0] + torch.log(z))
        ent.append(torch.log(z) - torch.where(e > 0, e * (s - m), torch.zeros_like(s)).sum(1) / z)
        lp = torch.gather(s, 1, t.clamp(min=0)) - lse[-1][:, None]
        logp.append(torch.where(t < 0, torch.zeros_like(lp), lp))
        if k > 0:
            val, pos = _best(s, k)
            short = k - val.shape[1]
            val = torch.nn.functional.pad(val - lse[-1][:, None], (0, short), value=-INF)
            tv.append(val)
            ti.append(torch.nn.functional.pad(pos, (0, short), value=-1))
    out = dict(logp=torch.cat(logp), lse=torch.cat(lse), entropy=torch.cat(ent))
    if k > 0:
        out.update(top_logp=torch.cat(tv), top_ids=torch.cat(ti))
    return out


def _plain_logprob_grad(state):
    case = state["case"]
    q, x, bias, targets, scale = state["q"].float(), state["x"].float(), state["bias"], state["targets"], state["scale"]
    dq, dx, db = [], torch.zeros_like(x), torch.zeros(case["nb"], device="cuda")
    for a in range(0, q.shape[0], _step(case)):
        b = min(a + _step(case), q.shape[0])
        s = _scores(q[a:b], x, scale, bias)
        logp = s - state["lse"][a:b, None]
        p = torch.exp(logp)
        t = targets[a:b]
        gt = torch.where(t < 0, torch.zeros_like(state["g_logp"][a:b]), state["g_logp"][a:b])
        grad = p * -gt.sum(1, keepdim=True)
        if state["g_entropy"] is not None:
            inner = torch.where(p > 0, logp + state["entropy"][a:b, None], torch.zeros_like(p))
            grad -= state["g_entropy"][a:b, None] * p * inner
        grad.scatter_add_(1, t.clamp(min=0), gt)
        if bias is not None:
            grad = torch.where(bias == -INF, torch.zeros_like(grad), grad)
        dq.append(scale * (grad @ x))
        dx += scale * (grad.t() @ q[a:b])
        db += grad.sum(0)
    dt = state["q"].dtype
    return dict(dq=torch.cat(dq).to(dt), dx=dx.to(dt), dbias=db)


def _probed_lists(state, q):
    """The nprobe lists whose centroids are nearest to the queries (zeros behind their dk components)."""
    cent = state["centroids"]
    qp = torch.nn.functional.pad(q, (0, cent.shape[1] - q.shape[1]))
    dist = (cent * cent).sum(1) - 2.0 * (qp @ cent.t())
    return torch.sort(dist, dim=1, stable=True).indices[:, :state["case"]["nprobe"]]


def _visit(state):
    """Pieces of a pass: (first query, query past the last, keys, values, row numbers or None, validity or None),
    keys and values [rows, .] for all queries of the piece, or [queries, rows, .]."""
    case = state["case"]
    dk, v0, nq = case["dk"], case["v0"], case["nq"]
    if case["nprobe"] == 0:
        rows = _decode(state["centroids"], state["codebooks"], state["codes"], state["list_of"])
        ids = torch.arange(case["nb"], device="cuda")
        for a in range(0, nq, _step(case)):
            yield a, min(a + _step(case), nq), rows[:, :dk], rows[:, v0:], ids[None, :], None
        return
    size = torch.bincount(state["list_of"], minlength=case["nlist"])
    off = torch.cumsum(size, 0) - size
    longest = int(size.max())
    q = state["q"].float()
    step = max(1, PLAIN_ELEMENTS // (case["nprobe"] * longest * case["d"]))
    lane = torch.arange(longest, device="cuda")
    for a in range(0, nq, step):
        b = min(a + step, nq)
        lists = _probed_lists(state, q[a:b])
        valid = (lane < size[lists][:, :, None]).reshape(b - a, -1)
        pos = (off[lists][:, :, None] + lane).clamp(max=case["nb"] - 1).reshape(b - a, -1)
        rows = _decode(state["centroids"], state["codebooks"], state["codes"][pos.reshape(-1)],
                       state["list_of"][pos.reshape(-1)]).reshape(b - a, -1, case["d"])
        yield a, b, rows[:, :, :dk], rows[:, :, v0:], pos, valid


def _rows_scores(state, q, keys, ids, valid, a, b):
    s = q @ keys.t() if keys.dim() == 2 else torch.bmm(keys, q[:, :, None])[:, :, 0]
    s = s * state["scale"]
    if state["limits"] is not None:
        s = torch.where(ids < state["limits"][a:b, None], s, torch.full_like(s, -INF))
    if valid is not None:
        s = torch.where(valid, s, torch.full_like(s, -INF))
    return s


def _weighted(p, rows):
    return p @ rows if rows.dim() == 2 else torch.bmm(p[:, None, :], rows)[:, 0, :]


def _plain_attend(state):
    q = state["q"].float()
    out, lse = [], []
    for a, b, keys, values, ids, valid in _visit(state):
        s = _rows_scores(state, q[a:b], keys, ids, valid, a, b)
        m = s.amax(1, keepdim=True)
        e = torch.exp(s - torch.where(m == -INF, torch.zeros_like(m), m))
        z = e.sum(1, keepdim=True)
        o = _weighted(e, values) / torch.where(z == 0, torch.ones_like(z), z)
        out.append(o)
        lse.append((m + torch.log(z))[:, 0])
    return dict(out=torch.cat(out).to(state["q"].dtype), lse=torch.cat(lse))


def _attend_lse(state):
    return _plain_attend(state)["lse"]


def _plain_attend_grad(state):
    q, g = state["q"].float(), state["g_out"].float()
    dq = []
    for a, b, keys, values, ids, valid in _visit(state):
        s = _rows_scores(state, q[a:b], keys, ids, valid, a, b)
        z = state["lse"][a:b, None]
        p = torch.exp(s - torch.where(z == -INF, torch.zeros_like(z), z))
        dp = g[a:b] @ values.t() if values.dim() == 2 else torch.bmm(values, g[a:b][:, :, None])[:, :, 0]
        ds = p * (dp - (p * dp).sum(1, keepdim=True))
        dq.append(state["scale"] * _weighted(ds, keys))
    return dict(dq=torch.cat(dq).to(state["q"].dtype))


# ---- one pass ------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if not own:
        return {"logprob": _plain_logprob, "logprob_grad": _plain_logprob_grad, "attend": _plain_attend,
                "attend_grad": _plain_attend_grad}[case["op"]](state)
    import paper_2401_08281_amd as vs
    if case["op"] == "logprob":
        logp, lse, ent, tv, ti = vs.vs_flat_logprob(state["x"], state["q"], state["targets"], case["k"],
                                                    scale=state["scale"], bias=state["bias"])
        out = dict(logp=logp, lse=lse, entropy=ent)
        if case["k"] > 0:
            out.update(top_logp=tv, top_ids=ti)
        return out
    if case["op"] == "logprob_grad":
        dx, dq, db = vs.vs_flat_logprob_grad(state["x"], state["q"], state["lse"], state["targets"], state["g_logp"],
                                             entropy=state["entropy"], g_entropy=state["g_entropy"],
                                             scale=state["scale"], bias=state["bias"])
        return dict(dq=dq, dx=dx, dbias=db)
    ix = state["index"]
    if case["op"] == "attend":
        out, lse = ix.attend(state["q"], case["nprobe"], state["scale"], v0=case["v0"], limits=state["limits"])
        return dict(out=out, lse=lse)
    return dict(dq=ix.attend_grad(state["q"], case["nprobe"], state["scale"], state["lse"], state["g_out"],
                                  v0=case["v0"], limits=state["limits"]))


def work(case):
    """Bytes that have to be moved and operations that have to be done.  Attention over codes: every byte of the
    visited codes once (lists that several queries share count once), per query and visited row one addition per
    key sub-quantizer, one per value sub-quantizer, and for the tables 2 x 16 operations per query component."""
    size = {"fp32": 4, "fp16": 2, "bf16": 2}[case["dtype"]]
    nq, nb, d = case["nq"], case["nb"], case["d"]
    if case["op"] == "logprob":
        return {"bytes": (nq + nb) * d * size + 8 * nq * case["nt"] + 4 * nq * (case["nt"] + 2) + 12 * nq * case["k"]
                + (4 * nb if case["bias"] != "none" else 0), "flops": 2 * nq * nb * d}
    if case["op"] == "logprob_grad":
        return {"bytes": 2 * (nq + nb) * d * size + 12 * nq * case["nt"] + 8 * nq
                + (4 * nb if case["bias"] != "none" else 0) + 4 * nb, "flops": 6 * nq * nb * d}
    share = case["nprobe"] / case["nlist"] if case["nprobe"] else 1.0
    rows = min(nb, nb * share * nq)
    pairs = nq * nb * share * (0.5 if case["limits"] else 1.0)
    dsub = d // case["M"]
    mk, mv = case["dk"] // dsub, (d - case["v0"]) // dsub
    out = nq * (d - case["v0"]) * size
    if case["op"] == "attend":
        return {"bytes": int(rows * case["M"] / 2 + nq * case["dk"] * size + out + 4 * nq),
                "flops": int(pairs * (mk + mv) + 32 * nq * (case["dk"] + d - case["v0"]))}
    return {"bytes": int(rows * case["M"] / 2 + 2 * nq * case["dk"] * size + out + 4 * nq),
            "flops": int(pairs * (2 * mk + mv) + 32 * nq * (2 * case["dk"] + d - case["v0"]))}


# ---- the definition in 64 bits ---------------------------------------------------------------------

def exact(case, seed):
    saved = globals()["own"]
    globals()["own"] = False
    try:
        state = prepare(case, seed)
    finally:
        globals()["own"] = saved
    return (_exact_logprob if case["op"].startswith("logprob") else _exact_attend)(case, state)


def _exact_logprob(case, st):
    nq, nb = case["nq"], case["nb"]
    x, q = st["x"].double(), st["q"].double()
    b = torch.zeros(nb, device="cuda", dtype=torch.float64) if st["bias"] is None else st["bias"].double()
    step = max(1, (1 << 26) // nb)
    parts, dx, db = [], torch.zeros_like(x), torch.zeros_like(b)
    for i in range(0, nq, step):
        j = min(i + step, nq)
        s = torch.addmm(b, q[i:j], x.t(), alpha=st["scale"])
        lp = torch.log_softmax(s, dim=1)
        p = lp.exp()
        plogp = torch.special.entr(p)
        t = st["targets"][i:j]
        if case["op"] == "logprob":
            row = dict(logp=torch.where(t >= 0, lp.gather(1, t.clamp(min=0)), 0.0), lse=torch.logsumexp(s, 1),
                       entropy=plogp.sum(1))
            if case["k"]:
                n = min(case["k"], nb)
                v, ids = torch.sort(lp, dim=1, descending=True, stable=True)
                row["top_logp"] = torch.full((j - i, case["k"]), -INF, device="cuda", dtype=torch.float64)
                row["top_ids"] = torch.full((j - i, case["k"]), -1, device="cuda", dtype=torch.int64)
                row["top_logp"][:, :n] = v[:, :n]
                row["top_ids"][:, :n] = torch.where(v[:, :n] > -INF, ids[:, :n], -1)
            parts.append(row)
            continue
        # d loss / d score through log-softmax: the cotangent of logp, minus p times its row sum
        cot = torch.zeros_like(s).scatter_add_(1, t.clamp(min=0), torch.where(t >= 0, st["g_logp"][i:j].double(), 0.0))
        if st["g_entropy"] is not None:
            # H = -sum p logp; its cotangent on logp is -(p logp + p)
            cot = cot + st["g_entropy"][i:j, None].double() * (plogp - p)
        grad = cot - p * cot.sum(1, keepdim=True)
        grad[:, b == -INF] = 0.0
        parts.append(dict(dq=st["scale"] * (grad @ x)))
        dx += st["scale"] * (grad.t() @ q[i:j])
        db += grad.sum(0)
    out = {name: torch.cat([r[name] for r in parts]) for name in parts[0]}
    if case["op"] == "logprob_grad":
        out.update(dx=dx, dbias=db)
    return out


def _exact_attend(case, st):
    nq, d, M, dk, v0 = case["nq"], case["d"], case["M"], case["dk"], case["v0"]
    dsub = d // M
    cent, books = st["centroids"].double(), st["codebooks"].double()
    vec = torch.empty(case["nb"], d, device="cuda", dtype=torch.float64)
    for m in range(M):
        byte = st["codes"][:, m // 2].long()
        c = (byte // 16) if m % 2 else (byte % 16)
        vec[:, m * dsub:(m + 1) * dsub] = books[m][c] + cent[:, m * dsub:(m + 1) * dsub][st["list_of"]]
    q = st["q"].double()
    first = torch.searchsorted(st["list_of"], torch.arange(case["nlist"] + 1, device="cuda")).tolist()
    if case["nprobe"]:
        gap = ((torch.nn.functional.pad(q, (0, d - dk))[:, None, :] - cent[None]) ** 2).sum(2) if case["nlist"] * nq * d < 1 << 28 \
            else torch.stack([((torch.nn.functional.pad(r, (0, d - dk)) - cent) ** 2).sum(1) for r in q])
        lists = torch.sort(gap, dim=1, stable=True).indices[:, :case["nprobe"]].tolist()
    out = torch.zeros(nq, d - v0, device="cuda", dtype=torch.float64)
    lse = torch.full((nq,), -INF, device="cuda", dtype=torch.float64)
    dq = torch.zeros(nq, dk, device="cuda", dtype=torch.float64)
    step = 1 if case["nprobe"] else max(1, (1 << 26) // case["nb"])
    limits = None if st["limits"] is None else st["limits"]
    for i in range(0, nq, step):
        j = min(i + step, nq)
        if case["nprobe"]:
            rows = torch.cat([torch.arange(first[l], first[l + 1], device="cuda") for l in lists[i]])
            x = vec[rows]
        else:
            rows, x = torch.arange(case["nb"], device="cuda"), vec
        if rows.numel() == 0:
            continue
        s = st["scale"] * (q[i:j] @ x[:, :dk].t())
        if limits is not None:
            s[rows[None, :] >= limits[i:j, None]] = -INF
        z = torch.logsumexp(s, 1)
        lse[i:j] = z
        p = torch.softmax(s, 1)
        p[z == -INF] = 0.0
        if case["op"] == "attend":
            out[i:j] = p @ x[:, v0:]
        else:
            gv = st["g_out"][i:j].double() @ x[:, v0:].t()
            mean = (p * gv).sum(1, keepdim=True)
            dq[i:j] = st["scale"] * ((p * (gv - mean)) @ x[:, :dk])
    return dict(out=out, lse=lse) if case["op"] == "attend" else dict(dq=dq)

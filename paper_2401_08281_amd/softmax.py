"""ctypes binding of libvs_softmax.so: same names as the C ABI in include/vs_softmax.h.

Argument marshalling only, as in binding.py.  Work space comes from torch's allocator, on the current
stream of the tensors' device, so a call can be captured into a graph (of attention: as long as nothing is
added to the index).  Nothing here is recorded by torch's autograd, whatever its tensors require: results
are leaves, and a training loop calls the *_grad functions, which return gradients.
"""
import ctypes
import os

import torch

from . import binding
from .binding import VSError, _dev, _p

VS_FP32, VS_FP16, VS_BF16 = 0, 1, 2
VS_MAX_TOP = 64

_DTYPES = {torch.float32: VS_FP32, torch.float16: VS_FP16, torch.bfloat16: VS_BF16}
_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libvs_softmax.so")
_lib = None


def softmax_lib():
    """Loads libvs_softmax.so, building it first if it is missing or older than one of its sources
    (VS_NO_REBUILD=1 in the environment loads a stale library as it is)."""
    global _lib
    if _lib is not None:
        return _lib
    binding.lib()
    from . import build
    if not os.path.exists(_LIB_PATH) or (build.softmax_is_stale() and os.environ.get("VS_NO_REBUILD") != "1"):
        build.build_softmax_lib()
    L = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    L.vs_flat_logprob_workspace_bytes.restype = i64
    L.vs_flat_logprob_workspace_bytes.argtypes = [i64, i64, i32, i32, i32]
    L.vs_flat_logprob.restype = ctypes.c_int
    L.vs_flat_logprob.argtypes = [vp, i64, vp, i64, i32, i32, f32, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, i64, vp]
    L.vs_flat_logprob_grad_workspace_bytes.restype = i64
    L.vs_flat_logprob_grad_workspace_bytes.argtypes = [i64, i64, i32, i32]
    L.vs_flat_logprob_grad.restype = ctypes.c_int
    L.vs_flat_logprob_grad.argtypes = [vp, i64, vp, i64, i32, i32, f32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
    L.vs_ivfpq_attend_workspace_bytes.restype = i64
    L.vs_ivfpq_attend_workspace_bytes.argtypes = [vp, i64, i32, i32, i32, i32]
    L.vs_ivfpq_attend.restype = ctypes.c_int
    L.vs_ivfpq_attend.argtypes = [vp, vp, i64, i32, i32, i32, i32, f32, vp, vp, vp, vp, i64, vp]
    L.vs_ivfpq_attend_grad_workspace_bytes.restype = i64
    L.vs_ivfpq_attend_grad_workspace_bytes.argtypes = [vp, i64, i32, i32, i32, i32]
    L.vs_ivfpq_attend_grad.restype = ctypes.c_int
    L.vs_ivfpq_attend_grad.argtypes = [vp, vp, i64, i32, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp, i64, vp]
    L.vs_softmax_last_error.restype = ctypes.c_char_p
    L.vs_softmax_last_error.argtypes = []
    _lib = L
    return L


def vs_softmax_last_error():
    return softmax_lib().vs_softmax_last_error().decode()


def _check(rc):
    if rc != 0:
        raise VSError(rc, vs_softmax_last_error())


def _space(n, device):
    # (arguments without a size are refused by the call itself, with the reason's code)
    return torch.empty(max(n, 0), dtype=torch.uint8, device=device)


def _vectors(t, name, like=None):
    """A 2-d device tensor of a vector type; `like`: of the same type and device as this one."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError("%s must be a device tensor" % name)
    if t.dtype not in _DTYPES:
        raise TypeError("%s must be float32, float16 or bfloat16, got %s" % (name, t.dtype))
    if t.dim() != 2:
        raise ValueError("%s must have two dimensions" % name)
    if like is not None and t.dtype != like.dtype:
        raise TypeError("%s must be %s, got %s" % (name, like.dtype, t.dtype))
    t = _on(t, name, like)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t if t.data_ptr() % 16 == 0 else t.clone()      # (rows cut out of a tensor may start anywhere)


def _on(t, name, like):
    if t is not None and like is not None and t.device != like.device:
        raise ValueError("%s is on %s, not on %s" % (name, t.device, like.device))
    return t


def _array(t, dtype, shape, name, like):
    if t is None:
        return None
    _on(_dev(t, dtype, name), name, like)
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s must be %s, got %s" % (name, list(shape), list(t.shape)))
    return t


def _stream_of(t):
    return ctypes.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)


def vs_flat_logprob_workspace_bytes(nb, nq, d, dtype, k):
    """Bytes of work space of one vs_flat_logprob (host arithmetic only); dtype: VS_FP32, VS_FP16 or VS_BF16."""
    n = int(softmax_lib().vs_flat_logprob_workspace_bytes(int(nb), int(nq), int(d), int(dtype), int(k)))
    if n < 0:
        raise VSError(-1, vs_softmax_last_error())
    return n


def vs_flat_logprob_grad_workspace_bytes(nb, nq, d, dtype):
    """Bytes of work space of one vs_flat_logprob_grad (host arithmetic only)."""
    n = int(softmax_lib().vs_flat_logprob_grad_workspace_bytes(int(nb), int(nq), int(d), int(dtype)))
    if n < 0:
        raise VSError(-1, vs_softmax_last_error())
    return n


def _rows_args(x, q, targets, bias):
    x = _vectors(x, "x")
    q = _vectors(q, "q", x)
    if q.shape[1] != x.shape[1]:
        raise ValueError("x and q differ in dimension")
    bias = _array(bias, torch.float32, (x.shape[0],), "bias", x)
    if targets is not None:
        _on(_dev(targets, torch.int64, "targets"), "targets", x)
        if targets.dim() != 2 or targets.shape[0] != q.shape[0]:
            raise ValueError("targets must be [nq, nt]")
    return x, q, targets, bias, 0 if targets is None else targets.shape[1]


def vs_flat_logprob(x, q, targets=None, k=0, scale=1.0, bias=None):
    """(logp [nq, nt], lse [nq], entropy [nq], top_logp [nq, k], top_ids [nq, k]) under the softmax of
    scale <q_i, x_j> + bias_j over the rows of x [nb, d]; x and q fp32, fp16 or bf16."""
    x, q, targets, bias, nt = _rows_args(x, q, targets, bias)
    (nb, d), nq, k = x.shape, q.shape[0], int(k)
    f32 = dict(dtype=torch.float32, device=x.device)
    with torch.cuda.device(x.device):
        logp = torch.empty((nq, nt), **f32)
        lse, entropy = torch.empty(nq, **f32), torch.empty(nq, **f32)
        top_logp = torch.empty((nq, max(k, 0)), **f32)
        top_ids = torch.empty((nq, max(k, 0)), dtype=torch.int64, device=x.device)
        ws = _space(softmax_lib().vs_flat_logprob_workspace_bytes(nb, nq, d, _DTYPES[x.dtype], k), x.device)
        _check(softmax_lib().vs_flat_logprob(_p(x), nb, _p(q), nq, d, _DTYPES[x.dtype], scale, _p(bias), _p(targets), nt,
                                             k, _p(logp), _p(lse), _p(entropy), _p(top_logp), _p(top_ids), _p(ws),
                                             ws.numel(), _stream_of(x)))
    return logp, lse, entropy, top_logp, top_ids


def vs_flat_logprob_grad(x, q, lse, targets=None, g_logp=None, g_lse=None, entropy=None, g_entropy=None, scale=1.0,
                         bias=None, want_dx=True, want_dq=True, want_dbias=True):
    """(dx, dq, dbias) of a loss whose gradients for vs_flat_logprob's outputs are g_logp [nq, nt], g_lse [nq] and
    g_entropy [nq] (None: zero); lse and entropy as vs_flat_logprob returned them.  dx and dq have the type of x and q;
    what is not wanted comes back as None."""
    x, q, targets, bias, nt = _rows_args(x, q, targets, bias)
    (nb, d), nq = x.shape, q.shape[0]
    lse = _array(lse, torch.float32, (nq,), "lse", x)
    entropy = _array(entropy, torch.float32, (nq,), "entropy", x)
    g_logp = _array(g_logp, torch.float32, (nq, nt), "g_logp", x)
    g_lse = _array(g_lse, torch.float32, (nq,), "g_lse", x)
    g_entropy = _array(g_entropy, torch.float32, (nq,), "g_entropy", x)
    if lse is None:
        raise TypeError("lse must be a device tensor")
    with torch.cuda.device(x.device):
        dx = torch.empty_like(x) if want_dx else None
        dq = torch.empty_like(q) if want_dq else None
        db = torch.empty(nb, dtype=torch.float32, device=x.device) if want_dbias else None
        ws = _space(softmax_lib().vs_flat_logprob_grad_workspace_bytes(nb, nq, d, _DTYPES[x.dtype]), x.device)
        _check(softmax_lib().vs_flat_logprob_grad(_p(x), nb, _p(q), nq, d, _DTYPES[x.dtype], scale, _p(bias), _p(targets),
                                                  nt, _p(lse), _p(entropy), _p(g_logp), _p(g_lse), _p(g_entropy), _p(dq),
                                                  _p(dx), _p(db), _p(ws), ws.numel(), _stream_of(x)))
    return dx, dq, db


def vs_ivfpq_attend_workspace_bytes(h, nq, dk, v0, dtype, nprobe):
    """Bytes of work space of one vs_ivfpq_attend on this index as it is."""
    n = int(softmax_lib().vs_ivfpq_attend_workspace_bytes(h, int(nq), int(dk), int(v0), int(dtype), int(nprobe)))
    if n < 0:
        raise VSError(-1, vs_softmax_last_error())
    return n


def vs_ivfpq_attend_grad_workspace_bytes(h, nq, dk, v0, dtype, nprobe):
    """Bytes of work space of one vs_ivfpq_attend_grad on this index as it is."""
    n = int(softmax_lib().vs_ivfpq_attend_grad_workspace_bytes(h, int(nq), int(dk), int(v0), int(dtype), int(nprobe)))
    if n < 0:
        raise VSError(-1, vs_softmax_last_error())
    return n


def vs_ivfpq_attend(h, d, q, nprobe, scale, v0=0, limits=None):
    """(out [nq, d - v0], lse [nq]): attention of q [nq, dk] over the vectors of a 4-bit IVF-PQ index of dimension d
    (keys: components [0, dk), values: [v0, d)), all of them (nprobe = 0) or those of the probed lists; query i sees
    ids below limits[i]."""
    q = _vectors(q, "q")
    nq, dk = q.shape
    limits = _array(limits, torch.int64, (nq,), "limits", q)
    with torch.cuda.device(q.device):
        out = torch.empty((nq, max(d - v0, 0)), dtype=q.dtype, device=q.device)
        lse = torch.empty(nq, dtype=torch.float32, device=q.device)
        ws = _space(softmax_lib().vs_ivfpq_attend_workspace_bytes(h, nq, dk, v0, _DTYPES[q.dtype], nprobe), q.device)
        _check(softmax_lib().vs_ivfpq_attend(h, _p(q), nq, dk, v0, _DTYPES[q.dtype], nprobe, scale, _p(limits), _p(out),
                                             _p(lse), _p(ws), ws.numel(), _stream_of(q)))
    return out, lse


def vs_ivfpq_attend_grad(h, d, q, nprobe, scale, lse, g_out, g_lse=None, v0=0, limits=None):
    """The gradient [nq, dk] for q of a loss whose gradients for vs_ivfpq_attend's outputs are g_out [nq, d - v0] and
    g_lse [nq] (None: zero); lse as vs_ivfpq_attend returned it."""
    q = _vectors(q, "q")
    nq, dk = q.shape
    limits = _array(limits, torch.int64, (nq,), "limits", q)
    lse = _array(lse, torch.float32, (nq,), "lse", q)
    g_out = _vectors(g_out, "g_out", q)
    g_lse = _array(g_lse, torch.float32, (nq,), "g_lse", q)
    if tuple(g_out.shape) != (nq, d - v0):
        raise ValueError("g_out must be [nq, d - v0]")
    with torch.cuda.device(q.device):
        dq = torch.empty_like(q)
        ws = _space(softmax_lib().vs_ivfpq_attend_grad_workspace_bytes(h, nq, dk, v0, _DTYPES[q.dtype], nprobe), q.device)
        _check(softmax_lib().vs_ivfpq_attend_grad(h, _p(q), nq, dk, v0, _DTYPES[q.dtype], nprobe, scale, _p(limits),
                                                  _p(lse), _p(g_out), _p(g_lse), _p(dq), _p(ws), ws.numel(), _stream_of(q)))
    return dq

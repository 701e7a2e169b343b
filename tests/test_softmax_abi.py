"""Host-side checks of libvs_softmax that need no GPU: the library exports what its header declares, the
binding has a function for every entry point, and bad arguments are refused before any device work."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "vs_softmax.h")
INVALID, UNSUPPORTED = -1, -2
NUL = ctypes.c_void_p(0)
ONE = ctypes.c_void_p(256)   # never dereferenced: validation fails first

BOUNDARY = """
vs_flat_logprob_workspace_bytes vs_flat_logprob vs_flat_logprob_grad_workspace_bytes vs_flat_logprob_grad
vs_ivfpq_attend_workspace_bytes vs_ivfpq_attend vs_ivfpq_attend_grad_workspace_bytes vs_ivfpq_attend_grad
vs_softmax_last_error
""".split()


@pytest.fixture(scope="module")
def L():
    import paper_2401_08281_amd as vs
    return vs.softmax_lib()


def declared_symbols():
    return re.findall(r"VS_API\s+[\w\s\*]+?\b(vs_\w+)\s*\(", open(HEADER).read())


def test_header_declares_the_boundary_and_the_library_exports_it(L):
    import paper_2401_08281_amd as vs
    import paper_2401_08281_amd.build as b
    assert sorted(declared_symbols()) == sorted(BOUNDARY)
    out = subprocess.run(["nm", "-D", "--defined-only", b.softmax_lib_path()], capture_output=True, text=True).stdout
    assert sorted(l.split()[-1] for l in out.splitlines() if " T " in l) == sorted(BOUNDARY)
    for name in BOUNDARY:
        assert callable(getattr(vs, name)), name


def logprob(L, x=ONE, nb=10, q=ONE, nq=2, d=8, dtype=0, scale=1.0, bias=NUL, targets=NUL, nt=0, k=0, logp=NUL, lse=ONE,
            ent=ONE, tv=NUL, ti=NUL, ws=ONE, n=1 << 40):
    return L.vs_flat_logprob(x, nb, q, nq, d, dtype, scale, bias, targets, nt, k, logp, lse, ent, tv, ti, ws, n, NUL)


@pytest.mark.parametrize("kw,text", [
    (dict(d=0), b"d = 0"), (dict(nb=-1), b"nb"), (dict(nb=1 << 31), b"nb"), (dict(nq=-1), b"nq"), (dict(dtype=3), b"dtype"),
    (dict(nt=-1), b"nt"), (dict(k=-1), b"k = -1"), (dict(k=65), b"k = 65"), (dict(scale=float("inf")), b"scale"),
    (dict(scale=float("nan")), b"scale"), (dict(x=NUL), b"null"), (dict(q=NUL), b"null"), (dict(lse=NUL), b"null"),
    (dict(ent=NUL), b"null"), (dict(nt=1, logp=ONE), b"null"), (dict(nt=1, targets=ONE), b"null"), (dict(k=1), b"null"),
    (dict(x=ctypes.c_void_p(8)), b"aligned"), (dict(q=ctypes.c_void_p(264)), b"aligned"), (dict(ws=NUL), b"work space"),
    (dict(ws=ctypes.c_void_p(128)), b"aligned"), (dict(n=0), b"work space"),
], ids=str)
def test_logprob_refuses(L, kw, text):
    assert logprob(L, **kw) == INVALID
    assert text in L.vs_softmax_last_error()


def test_no_queries_is_no_work(L):
    assert logprob(L, nq=0, x=NUL, q=NUL, lse=NUL, ent=NUL, ws=NUL, n=0) == 0
    assert L.vs_flat_logprob_workspace_bytes(10, 0, 8, 0, 5) == 0
    assert L.vs_flat_logprob_grad_workspace_bytes(10, 0, 8, 0) == 0
    assert L.vs_flat_logprob_grad_workspace_bytes(0, 10, 8, 0) == 0


def grad(L, x=ONE, nb=10, q=ONE, nq=2, d=8, dtype=0, scale=1.0, targets=NUL, nt=0, lse=ONE, ent=NUL, gl=NUL, ge=NUL, dq=ONE,
         dx=ONE, db=ONE, ws=ONE, n=1 << 40):
    return L.vs_flat_logprob_grad(x, nb, q, nq, d, dtype, scale, NUL, targets, nt, lse, ent, gl, NUL, ge, dq, dx, db, ws, n, NUL)


@pytest.mark.parametrize("kw,text", [
    (dict(d=0), b"d = 0"), (dict(nb=1 << 31), b"nb"), (dict(nq=-1), b"nq"), (dict(dtype=-1), b"dtype"), (dict(nt=-1), b"nt"),
    (dict(scale=float("inf")), b"scale"), (dict(x=NUL), b"null"), (dict(q=NUL), b"null"), (dict(lse=NUL), b"null"),
    (dict(nt=1, gl=ONE), b"null"), (dict(ge=ONE), b"entropy"), (dict(x=ctypes.c_void_p(8)), b"aligned"),
    (dict(dq=ctypes.c_void_p(2)), b"aligned"), (dict(ws=NUL), b"work space"), (dict(n=100), b"work space"),
], ids=str)
def test_logprob_grad_refuses(L, kw, text):
    assert grad(L, **kw) == INVALID
    assert text in L.vs_softmax_last_error()


def test_workspace_functions_refuse(L):
    import paper_2401_08281_amd as vs
    for args in ((-1, 1, 8, 0, 0), (1, 1, 0, 0, 0), (1, 1, 8, 9, 0), (1, 1, 8, 0, 65)):
        with pytest.raises(vs.VSError):
            vs.vs_flat_logprob_workspace_bytes(*args)
    with pytest.raises(vs.VSError):
        vs.vs_flat_logprob_grad_workspace_bytes(1, 1 << 31, 8, 0)


def test_work_space_stays_bounded():
    """Scores and gradients are never held for all pairs: a piece of the queries or rows at a time."""
    import paper_2401_08281_amd as vs
    for dtype, size in ((0, 4), (1, 2), (2, 2)):
        for nb, nq, d in ((1_000_000, 10_000, 128), (65_536, 65_536, 768), (10_000_000, 100, 96)):
            copies = 4 * (nb + nq) * (d + 32) * size          # both operands, by rows and by columns, in 16-bit parts
            parts = (nb + 127) // 128 * 16 * 128
            assert vs.vs_flat_logprob_workspace_bytes(nb, nq, d, dtype, 0) <= copies + parts + (300 << 20)
            sums = 16 * (nq + 200_000) * (d + 4) * 4
            assert vs.vs_flat_logprob_grad_workspace_bytes(nb, nq, d, dtype) <= copies + sums + (600 << 20)


def test_attend_refuses_without_an_index(L):
    assert L.vs_ivfpq_attend(NUL, ONE, 1, 8, 0, 0, 0, 1.0, NUL, ONE, ONE, ONE, 1 << 30, NUL) == INVALID
    assert b"index is null" in L.vs_softmax_last_error()
    assert L.vs_ivfpq_attend_grad(NUL, ONE, 1, 8, 0, 0, 0, 1.0, NUL, ONE, ONE, NUL, ONE, ONE, 1 << 30, NUL) == INVALID
    assert L.vs_ivfpq_attend_workspace_bytes(NUL, 1, 8, 0, 0, 0) == -1
    assert L.vs_ivfpq_attend_grad_workspace_bytes(NUL, 1, 8, 0, 0, 0) == -1


def test_binding_refuses_host_tensors_and_other_types():
    import torch
    import paper_2401_08281_amd as vs
    with pytest.raises(TypeError):
        vs.vs_flat_logprob(torch.zeros(4, 2), torch.zeros(1, 2))
    with pytest.raises(TypeError):
        vs.vs_flat_logprob_grad(torch.zeros(4, 2), torch.zeros(1, 2), torch.zeros(1))
    with pytest.raises(TypeError):
        vs.vs_ivfpq_attend(None, 2, torch.zeros(1, 2), 0, 1.0)

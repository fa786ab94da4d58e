"""CPU checks of include/mv_lm.h: workspace sizes and the refusals that happen before anything is enqueued."""
import ctypes
import math

import pytest

from paper_2011_06495_b200 import binding as B
from paper_2011_06495_b200 import build as BUILD


@pytest.fixture(scope="module")
def lib():
    BUILD.build()
    return B.load()


P = ctypes.c_void_p(0x100000)          # never dereferenced
Q = ctypes.c_void_p(0x200000)
R = ctypes.c_void_p(0x300000)
ODD = ctypes.c_void_p(0x100002)
BAD = B.MV_ERR_INVALID_ARG


def test_embed_refusals(lib):
    ok = dict(w=P, wt=B.MV_F32, V=10, D=8, ldw=8, ids=Q, it=B.MV_I64, T=4, out=R, ot=B.MV_BF16, ldo=8)

    def call(**k):
        a = {**ok, **k}
        return lib.mv_embed(None, a["w"], a["wt"], a["V"], a["D"], a["ldw"], a["ids"], a["it"], a["T"], 1.0, a["out"], a["ot"], a["ldo"])

    for k in (dict(w=None), dict(wt=B.MV_I32), dict(wt=9), dict(V=0), dict(V=1 << 31), dict(D=0), dict(ldw=7), dict(ids=None), dict(it=B.MV_F32),
              dict(T=-1), dict(T=1 << 31), dict(out=None), dict(ot=5), dict(ldo=7), dict(w=ODD), dict(ids=ODD), dict(ids=ctypes.c_void_p(0x100004)), dict(out=P), dict(out=ctypes.c_void_p(0x100000 - 62)),
              dict(out=ctypes.c_void_p(0x100000 + 318))):
        assert call(**k) == BAD, k
    assert call(T=0) == B.MV_OK


def test_embed_grad_refusals_and_workspace(lib):
    need = B.embed_grad_workspace_bytes(1000, 50, 8)
    assert need >= 8000 and need % 16 == 0
    assert B.embed_grad_workspace_bytes(-1, 50, 8) == 0 and B.embed_grad_workspace_bytes(10, 0, 8) == 0 and B.embed_grad_workspace_bytes(10, 50, 1 << 31) == 0
    assert B.embed_grad_workspace_bytes(0, 50, 8) > 0
    ok = dict(x=P, xt=B.MV_F16, ldd=8, ids=Q, it=B.MV_I32, T=1000, V=50, D=8, acc=0, dw=R, ldw=8, ws=Q, n=need)

    def call(**k):
        a = {**ok, **k}
        return lib.mv_embed_grad(None, a["x"], a["xt"], a["ldd"], a["ids"], a["it"], a["T"], a["V"], a["D"], 1.0, -1, a["acc"], a["dw"], a["ldw"], a["ws"], a["n"])

    for k in (dict(x=None), dict(xt=7), dict(ldd=7), dict(ids=None), dict(it=B.MV_BF16), dict(T=-1), dict(V=0), dict(D=0), dict(acc=2), dict(dw=None),
              dict(ldw=7), dict(dw=ODD), dict(ids=ODD), dict(x=ctypes.c_void_p(0x100001)), dict(ws=ctypes.c_void_p(0x100008)), dict(dw=P)):
        assert call(**k) == BAD, k
    assert call(ws=None) == B.MV_ERR_WORKSPACE and call(n=need - 1) == B.MV_ERR_WORKSPACE


def test_token_refusals(lib):
    ok = dict(x=P, xt=B.MV_BF16, T=4, V=30, ld=30, y=Q, it=B.MV_I64, c=1.0, k=0, lp=P, ent=None, lse=None, tl=None, ti=None)

    def call(**k):
        a = {**ok, **k}
        return lib.mv_token_logprob(None, a["x"], a["xt"], a["T"], a["V"], a["ld"], a["y"], a["it"], a["c"], a["k"], a["lp"], a["ent"], a["lse"], a["tl"], a["ti"])

    for k in (dict(x=None), dict(xt=3), dict(T=-1), dict(V=0), dict(V=1 << 31), dict(ld=29), dict(y=None), dict(it=0), dict(c=0.0), dict(c=-1.0),
              dict(c=math.inf), dict(c=math.nan), dict(k=-1), dict(k=65), dict(lp=ODD), dict(ti=ODD), dict(y=ODD), dict(x=ctypes.c_void_p(0x100001))):
        assert call(**k) == BAD, k
    assert call(T=0) == B.MV_OK

    okg = dict(x=P, xt=B.MV_F32, T=4, V=30, ld=30, y=Q, it=B.MV_I64, c=1.0, lse=Q, ent=Q, g1=Q, g2=Q, dx=ctypes.c_void_p(0x300000), ldg=30)

    def grad(**k):
        a = {**okg, **k}
        return lib.mv_token_logprob_grad(None, a["x"], a["xt"], a["T"], a["V"], a["ld"], a["y"], a["it"], a["c"], a["lse"], a["ent"], a["g1"], a["g2"], a["dx"], a["ldg"])

    for k in (dict(x=None), dict(lse=None), dict(dx=None), dict(ent=None), dict(y=None), dict(g1=None, g2=None), dict(ldg=29), dict(ld=29), dict(c=0.0),
              dict(dx=ctypes.c_void_p(0x100004)), dict(dx=P, ldg=31), dict(dx=ctypes.c_void_p(0x100000 - 40)), dict(it=1)):
        assert grad(**k) == BAD, k
    assert grad(T=0) == B.MV_OK


def test_clip_refusals_and_workspace(lib):
    n = (ctypes.c_int64 * 3)(100, 0, 50_000)
    need = lib.mv_clip_workspace_bytes(n, 3, 2)
    assert need > 0 and need % 256 == 0
    assert lib.mv_clip_workspace_bytes(n, -1, 1) == 0 and lib.mv_clip_workspace_bytes(n, 3, 0) == 0 and lib.mv_clip_workspace_bytes(None, 3, 1) == 0
    assert lib.mv_clip_workspace_bytes((ctypes.c_int64 * 1)(-1), 1, 1) == 0 and lib.mv_clip_workspace_bytes(None, 0, 1) > 0
    ptr = (ctypes.c_void_p * 3)(0x1000, 0, 0x200000)
    types = (ctypes.c_int * 3)(B.MV_F32, B.MV_F32, B.MV_BF16)
    groups = (ctypes.c_int * 3)(0, 1, 1)
    h = ctypes.c_void_p()

    def create(out=ctypes.byref(h), p=ptr, t=types, n=n, g=groups, nt=3, ng=2, ws=P, size=need):
        return lib.mv_clip_create(out, None, p, t, n, g, nt, ng, ws, size)

    assert create(out=None) == BAD and create(p=None) == BAD and create(t=None) == BAD and create(ng=0) == BAD
    assert create(ws=ctypes.c_void_p(0x100080)) == BAD
    assert create(p=(ctypes.c_void_p * 3)(0, 0, 0x200000)) == BAD and create(p=(ctypes.c_void_p * 3)(0x1002, 0, 0x200000)) == BAD
    assert create(t=(ctypes.c_int * 3)(0, 0, 4)) == BAD
    assert create(g=(ctypes.c_int * 3)(0, 1, 0)) == BAD and create(g=(ctypes.c_int * 3)(0, 1, 2)) == BAD and create(g=(ctypes.c_int * 3)(-1, 0, 0)) == BAD
    assert create(ws=None) == B.MV_ERR_WORKSPACE and create(size=need - 1) == B.MV_ERR_WORKSPACE
    assert not h
    assert lib.mv_clip_destroy(None) == BAD and lib.mv_clip_norm(None, None, P) == BAD
    assert lib.mv_clip_scale(None, None, 1.0, None) == BAD and lib.mv_clip_pack(None, None, 1.0, P, 10, None) == BAD

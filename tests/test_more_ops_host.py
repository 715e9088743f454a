"""Argument checks of packed arrays and layers, kept activations, block norms and sampling: host logic, no GPU."""
import ctypes
import os
import re

import pytest
import torch

import paper_2007_07336_amd as M
from paper_2007_07336_amd import binding as Bd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20               # aligned, never dereferenced: every call below is turned away before anything is launched
BIG = 1 << 60
E = Bd


@pytest.mark.parametrize("name", ["packed", "affine_packed", "block_norm", "sample"])
def test_structs_match_the_header(name):
    hdr = open(os.path.join(ROOT, "include", "mgrit.h")).read()
    body = re.sub(r"/\*.*?\*/", "", hdr[hdr.index("typedef struct mgrit_%s {" % name):hdr.index("} mgrit_%s_t;" % name)], flags=re.S)
    fields = []
    for kind, decl in re.findall(r"(int32_t|float)\s+([^;]+);", body):
        fields += [(f.strip(), {"int32_t": ctypes.c_int32, "float": ctypes.c_float}[kind]) for f in decl.split(",")]
    assert fields == list(getattr(Bd, "mgrit_%s_t" % name)._fields_)


def test_constants_match_the_header():
    hdr = open(os.path.join(ROOT, "include", "mgrit.h")).read()
    for name in ("MGRIT_MX8", "MGRIT_MX4", "MGRIT_NORM_ROOT", "MGRIT_NORM_LAYER", "MGRIT_GATE_NONE", "MGRIT_GATE_FEATURE", "MGRIT_GATE_ENTRY"):
        assert int(re.search(r"\b%s = (\d+)" % name, hdr).group(1)) == getattr(M, name)


# ---------------------------------------------------------------------------------------------- packed arrays
def _pack(p, X=FAKE, a=FAKE, back=False):
    L = M.lib()
    return L.mgrit_unpack(ctypes.byref(p) if p else None, a, X, None) if back else L.mgrit_pack(ctypes.byref(p) if p else None, X, a, None)


@pytest.mark.parametrize("back", [False, True])
def test_packed_arguments(back):
    new = lambda **kw: M.make_packed(**dict(dict(rows=3, cols=40, format=M.MGRIT_MX4), **kw))       # noqa: E731
    assert _pack(None, back=back) == E.MGRIT_ERR_POINTER and M.lib().mgrit_packed_bytes(None) == 0
    for bad in (dict(rows=-1), dict(cols=0), dict(format=0), dict(format=1), dict(format=5), dict(dtype=2), dict(dtype=M.MGRIT_MX8)):
        assert _pack(new(**bad), back=back) == E.MGRIT_ERR_PROBLEM and M.mgrit_packed_bytes(new(**bad)) == 0, bad
    big = new(rows=1 << 30, cols=257)
    assert _pack(big, back=back) == E.MGRIT_ERR_UNSUPPORTED and M.mgrit_packed_bytes(big) == 0
    p = new()
    for kw in (dict(X=None), dict(a=None), dict(X=FAKE + 8), dict(a=FAKE + 16)):
        assert _pack(p, back=back, **kw) == E.MGRIT_ERR_POINTER, kw
    assert _pack(new(rows=0), X=None, a=None, back=back) == E.MGRIT_OK


def test_packed_sizes():
    for rows, cols in ((1, 1), (3, 256), (3, 257), (7, 1031), (1 << 20, 4096)):
        slabs = (cols + 255) // 256
        for form, per in ((M.MGRIT_MX8, 256), (M.MGRIT_MX4, 128)):
            up = lambda n: (n + 255) // 256 * 256                                                    # noqa: E731
            assert M.mgrit_packed_bytes(M.make_packed(rows=rows, cols=cols, format=form)) == up(rows * slabs * per) + up(rows * slabs * 8)
    assert M.mgrit_packed_bytes(M.make_packed(rows=0, cols=5, format=M.MGRIT_MX8)) == 0


# ---------------------------------------------------------------------------------------------- layers with packed weights
def _fwd(p, X=FAKE, W=FAKE, b=None, R=None, Y=FAKE, D=None, ws=FAKE, n=BIG):
    return M.lib().mgrit_affine_packed_forward(ctypes.byref(p) if p else None, X, W, b, R, Y, D, ws, n, None)


def test_packed_layer_arguments():
    new = lambda **kw: M.make_affine_packed(**dict(dict(M=4, K=80, F=30), **kw))                     # noqa: E731
    assert _fwd(None) == E.MGRIT_ERR_POINTER
    for bad in (dict(M=-1), dict(K=0), dict(F=0), dict(act=3), dict(act=-1), dict(xtype=2), dict(xtype=M.MGRIT_MX4), dict(xformat=M.MGRIT_FP32),
                dict(xformat=M.MGRIT_MX8), dict(ytype=4), dict(scale=float("inf")), dict(scale=float("nan"))):
        assert _fwd(new(**bad)) == E.MGRIT_ERR_PROBLEM and M.mgrit_affine_packed_workspace_bytes(new(**bad)) == 0, bad
    for big in (dict(K=(1 << 22) + 1), dict(M=1 << 20, F=1 << 20), dict(F=1 << 30, K=300)):
        assert _fwd(new(**big)) == E.MGRIT_ERR_UNSUPPORTED and M.mgrit_affine_packed_workspace_bytes(new(**big)) == 0, big
    for form in (M.MGRIT_BF16, M.MGRIT_MX4):
        for rows in (4, 100, 1000):
            p = new(M=rows, xformat=form)
            n = M.mgrit_affine_packed_workspace_bytes(p)
            for k in ("X", "W", "Y"):
                assert _fwd(p, **{k: None}) == E.MGRIT_ERR_POINTER
            for k in ("X", "b", "R", "Y", "D", "ws"):
                assert _fwd(p, **{k: FAKE + 4}) == E.MGRIT_ERR_POINTER, k
            assert _fwd(p, W=FAKE + 16) == E.MGRIT_ERR_POINTER
            if n:
                assert _fwd(p, n=n - 1) == E.MGRIT_ERR_WORKSPACE and _fwd(p, ws=None) == E.MGRIT_ERR_POINTER
    assert _fwd(new(M=0), X=None, W=None, Y=None, ws=None, n=0) == E.MGRIT_OK


# ---------------------------------------------------------------------------------------------- kept activations
def _kept(p, X=FAKE, W=FAKE, D=None, dY=FAKE, dX=FAKE, dW=FAKE, db=FAKE, ws=FAKE, n=BIG):
    return M.lib().mgrit_affine_kept_backward(ctypes.byref(p) if p else None, X, W, D, dY, dX, dW, db, ws, n, None)


def test_kept_arguments():
    new = lambda **kw: M.make_affine(**dict(dict(M=40, K=80, F=30), **kw))                           # noqa: E731
    assert _kept(None) == E.MGRIT_ERR_POINTER
    for bad in (dict(M=-1), dict(K=0), dict(F=0), dict(act=3), dict(xtype=2), dict(wtype=M.MGRIT_MX4), dict(ytype=M.MGRIT_MX8), dict(scale=float("nan"))):
        assert _kept(new(**bad)) == E.MGRIT_ERR_PROBLEM and M.mgrit_affine_kept_workspace_bytes(new(**bad)) == 0, bad
    p = new()
    n = M.mgrit_affine_kept_workspace_bytes(p)
    assert n > 0 and _kept(p, n=n - 1) == E.MGRIT_ERR_WORKSPACE
    for kw in (dict(dY=None), dict(X=None), dict(W=None), dict(ws=None), dict(X=FAKE + 16), dict(D=FAKE + 16)):
        assert _kept(p, **kw) == E.MGRIT_ERR_POINTER, kw
    for k in ("W", "dY", "dX", "dW", "db", "ws"):
        assert _kept(p, **{k: FAKE + 4}) == E.MGRIT_ERR_POINTER, k
    assert _kept(new(act=M.MGRIT_ACT_TANH)) == E.MGRIT_ERR_POINTER                # only the identity does without factors
    assert _kept(p, dX=None, dW=None, db=None) == E.MGRIT_OK
    assert _kept(new(M=0), dW=None, db=None) == E.MGRIT_OK


# ---------------------------------------------------------------------------------------------- block norms
def _norm_fwd(p, f=FAKE, r=FAKE, gate=None, post=FAKE, pre=FAKE, S=FAKE, Y=FAKE):
    return M.lib().mgrit_block_norm_forward(ctypes.byref(p) if p else None, f, r, gate, post, pre, S, Y, None)


def _norm_bwd(p, f=FAKE, S=FAKE, gate=None, post=FAKE, pre=FAKE, dS=FAKE, dY=FAKE, df=FAKE, dr=FAKE, dgate=None, dpost=FAKE, dpre=FAKE, ws=FAKE, n=BIG):
    return M.lib().mgrit_block_norm_backward(ctypes.byref(p) if p else None, f, S, gate, post, pre, dS, dY, df, dr, dgate, dpost, dpre, ws, n, None)


def test_block_norm_arguments():
    new = lambda **kw: M.make_block_norm(**dict(dict(M=4, q=80), **kw))                              # noqa: E731
    assert _norm_fwd(None) == _norm_bwd(None) == E.MGRIT_ERR_POINTER
    for bad in (dict(M=-1), dict(q=0), dict(kind=2), dict(kind=-1), dict(gate=3), dict(stype=2), dict(ftype=-1), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(scale=float("inf"))):
        assert _norm_fwd(new(**bad)) == _norm_bwd(new(**bad)) == E.MGRIT_ERR_PROBLEM and M.mgrit_block_norm_workspace_bytes(new(**bad)) == 0, bad
    big = new(M=1 << 20, q=1 << 20)
    assert _norm_fwd(big) == _norm_bwd(big) == E.MGRIT_ERR_UNSUPPORTED
    p, g = new(), new(gate=M.MGRIT_GATE_FEATURE)
    for kw in (dict(f=None), dict(r=None), dict(S=None), dict(Y=None), dict(pre=None), dict(gate=FAKE)):
        assert _norm_fwd(p, **kw) == E.MGRIT_ERR_POINTER, kw
    assert _norm_fwd(g) == E.MGRIT_ERR_POINTER                                    # where is the gate
    for k in ("f", "r", "post", "pre", "S", "Y"):
        assert _norm_fwd(p, **{k: FAKE + 4}) == E.MGRIT_ERR_POINTER, k
    for kw in (dict(f=None), dict(S=None), dict(pre=None), dict(dY=None), dict(post=None), dict(gate=FAKE), dict(dgate=FAKE), dict(ws=None)):
        assert _norm_bwd(p, **kw) == E.MGRIT_ERR_POINTER, kw
    assert _norm_bwd(p, pre=None, dY=None) == E.MGRIT_ERR_POINTER                 # no such weights, but their gradient
    for k in ("f", "S", "post", "pre", "dS", "dY", "df", "dr", "dpost", "dpre", "ws"):
        assert _norm_bwd(p, **{k: FAKE + 4}) == E.MGRIT_ERR_POINTER, k
    n = M.mgrit_block_norm_workspace_bytes(p)
    assert n > 0 and _norm_bwd(p, n=n - 1) == E.MGRIT_ERR_WORKSPACE
    assert _norm_bwd(p, df=None, dr=None, dpost=None, dpre=None) == E.MGRIT_OK
    assert _norm_fwd(new(M=0), f=None, r=None, S=None, Y=None, pre=None) == E.MGRIT_OK


# ---------------------------------------------------------------------------------------------- sampling
def _sample(p, x=FAKE, u=FAKE, t=None, k=None, top=None, least=None, index=FAKE, logprob=None, ws=None, n=0):
    return M.lib().mgrit_sample(ctypes.byref(p) if p else None, x, u, t, k, top, least, index, logprob, ws, n, None)


def test_sample_arguments():
    assert _sample(None) == E.MGRIT_ERR_POINTER
    for bad in (dict(B=-1), dict(V=0), dict(dtype=2), dict(dtype=M.MGRIT_MX8)):
        assert _sample(M.make_sample(**dict(dict(B=4, V=10), **bad))) == E.MGRIT_ERR_PROBLEM, bad
    assert _sample(M.make_sample(B=1 << 30, V=1 << 10)) == E.MGRIT_ERR_UNSUPPORTED
    p = M.make_sample(B=4, V=10)
    n = M.mgrit_sample_workspace_bytes(p)
    for k in ("x", "u", "index"):
        assert _sample(p, ws=FAKE, n=n, **{k: None}) == E.MGRIT_ERR_POINTER, k
    for k in ("x", "u", "t", "k", "top", "least", "index", "logprob"):
        assert _sample(p, ws=FAKE, n=n, **{k: FAKE + 4}) == E.MGRIT_ERR_POINTER, k
    assert _sample(M.make_sample(B=0, V=10), x=None, u=None, index=None) == E.MGRIT_OK


# ---------------------------------------------------------------------------------------------- the binding
def test_binding_refuses_tensors_that_do_not_fit():
    p = M.make_packed(rows=3, cols=40, format=M.MGRIT_MX4)
    X, a = torch.zeros(3, 40), torch.zeros(M.mgrit_packed_bytes(p), dtype=torch.uint8)
    for args, word in (((X.bfloat16(), a), "X has type"), ((X[:, :39].contiguous(), a), "X has 117 values"), ((X, a[:-1]), "packed has"),
                       ((X, a.view(torch.int8)), "packed has type"), ((torch.zeros(40, 3).T, a), "not contiguous"), ((X, a), "not on a GPU")):
        with pytest.raises(ValueError, match=word):
            M.mgrit_pack(p, *args)
        with pytest.raises(ValueError, match=word):
            M.mgrit_unpack(p, args[1], args[0])
    f = M.make_affine_packed(M=2, K=40, F=3)
    with pytest.raises(ValueError, match="W has"):
        M.mgrit_affine_packed_forward(f, torch.zeros(2, 40), a[:-256], None, None, torch.zeros(2, 3), None, None)
    k = M.make_affine(M=3, K=40, F=5)
    with pytest.raises(ValueError, match="X has"):
        M.mgrit_affine_kept_backward(k, a, None, None, torch.zeros(3, 5), None, torch.zeros(5, 40), None, None)     # (packed, but not as MX8)
    n = M.make_block_norm(M=2, q=8, gate=M.MGRIT_GATE_FEATURE)
    with pytest.raises(ValueError, match="gate has 16 values"):
        M.mgrit_block_norm_forward(n, torch.zeros(2, 8), torch.zeros(2, 8), torch.zeros(2, 8), None, None, torch.zeros(2, 8), None)
    with pytest.raises(ValueError, match="dS has type"):
        M.mgrit_block_norm_backward(n, torch.zeros(2, 8), torch.zeros(2, 8), torch.zeros(8), None, None, torch.zeros(2, 8).double(), None, torch.zeros(2, 8),
                                    None, None, None, None, None)
    s = M.make_sample(B=2, V=8)
    with pytest.raises(ValueError, match="top_k has type"):
        M.mgrit_sample(s, torch.zeros(2, 8), torch.zeros(2), None, torch.ones(2, dtype=torch.int64), None, None, torch.zeros(2, dtype=torch.int64), None, None)
    with pytest.raises(ValueError, match="index has type"):
        M.mgrit_sample(s, torch.zeros(2, 8), torch.zeros(2), None, None, None, None, torch.zeros(2, dtype=torch.int32), None, None)


def test_the_operators_take_no_memory_on_the_host():
    csrc = os.path.join(ROOT, "paper_2007_07336_amd", "csrc")
    for name in ("mgrit_packed.hip", "mgrit_norm.hip", "mgrit_sample.hip", "mgrit_epilogue.h"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, name)).read())
        assert not re.search(r"\b(new|malloc|calloc|hipMalloc\w*|hipHostMalloc|std::(vector|string|map|unique_ptr|function|make_\w+))\b", text), name

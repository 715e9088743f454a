"""Argument checks of the operators around the solver (end layers, loss, clipping): host logic, no GPU."""
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


@pytest.mark.parametrize("name", ["affine", "loss", "tensor"])
def test_structs_match_the_header(name):
    hdr = open(os.path.join(ROOT, "include", "mgrit.h")).read()
    body = re.sub(r"/\*.*?\*/", "", hdr[hdr.index("typedef struct mgrit_%s {" % name):hdr.index("} mgrit_%s_t;" % name)], flags=re.S)
    fields = []
    for decl in re.findall(r"(?:int32_t|int64_t|float|void\*)\s+([^;]+);", body):
        fields += [f.strip() for f in decl.split(",")]
    assert fields == [f[0] for f in getattr(Bd, "mgrit_%s_t" % name)._fields_]


def _affine(**kw):
    return M.make_affine(**dict(dict(M=4, K=8, F=3), **kw))


def _fwd(p, X=FAKE, W=FAKE, b=None, R=None, Y=FAKE, D=None, ws=FAKE, n=0):
    return M.lib().mgrit_affine_forward(ctypes.byref(p) if p else None, X, W, b, R, Y, D, ws, n, None)


def _bwd(p, X=FAKE, W=FAKE, D=None, dY=FAKE, dX=FAKE, dW=FAKE, db=FAKE, ws=FAKE, n=0):
    return M.lib().mgrit_affine_backward(ctypes.byref(p) if p else None, X, W, D, dY, dX, dW, db, ws, n, None)


BAD = [dict(M=-1), dict(K=0), dict(F=0), dict(K=-5), dict(act=3), dict(act=-1), dict(xtype=2), dict(wtype=-1), dict(ytype=7),
       dict(scale=float("inf")), dict(scale=float("nan"))]


@pytest.mark.parametrize("bad", BAD)
def test_invalid_layers(bad):
    p = _affine(**bad)
    assert _fwd(p) == _bwd(p) == Bd.MGRIT_ERR_PROBLEM
    assert M.mgrit_affine_workspace_bytes(p) == M.mgrit_affine_backward_workspace_bytes(p) == 0


def test_layer_pointers_and_sizes():
    p = _affine()
    assert _fwd(None) == _bwd(None) == Bd.MGRIT_ERR_POINTER
    for k in ("X", "W", "Y"):
        assert _fwd(p, **{k: None}) == Bd.MGRIT_ERR_POINTER
    for k in ("X", "W", "b", "R", "Y", "D", "ws"):
        assert _fwd(p, **{k: FAKE + 4}) == Bd.MGRIT_ERR_POINTER, k
    assert _bwd(p, dY=None) == Bd.MGRIT_ERR_POINTER
    assert _bwd(p, X=None) == Bd.MGRIT_ERR_POINTER                  # dW wants it
    assert _bwd(p, W=None) == Bd.MGRIT_ERR_POINTER                  # dX wants it
    for k in ("X", "W", "D", "dY", "dX", "dW", "db", "ws"):
        assert _bwd(p, **{k: FAKE + 4}) == Bd.MGRIT_ERR_POINTER, k
    assert _bwd(_affine(act=M.MGRIT_ACT_TANH)) == Bd.MGRIT_ERR_POINTER     # only the identity does without factors
    big = _affine(M=1 << 20, K=1 << 20, F=1)
    assert _fwd(big, n=BIG) == _bwd(big, n=BIG) == Bd.MGRIT_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(M=32, K=65536, F=10), dict(M=512, K=512, F=512, xtype=1, wtype=1, ytype=1), dict(M=300, K=1111, F=777),
                                dict(M=2000, K=1024, F=10, wtype=1), dict(M=1, K=4096, F=512, xtype=1, wtype=1)])
def test_a_workspace_that_is_too_small(kw):
    p = _affine(**kw)
    n = M.mgrit_affine_workspace_bytes(p)
    if n:
        assert _fwd(p, n=n - 1) == Bd.MGRIT_ERR_WORKSPACE
        assert _fwd(p, ws=None, n=n) == Bd.MGRIT_ERR_POINTER
    n = M.mgrit_affine_backward_workspace_bytes(p)
    if n:
        assert _bwd(p, n=n - 1) == Bd.MGRIT_ERR_WORKSPACE
        assert _bwd(p, ws=None, n=n) == Bd.MGRIT_ERR_POINTER


def _ce(p, x=FAKE, y=FAKE, loss=FAKE, rows=FAKE, grad=FAKE, ws=FAKE, n=0):
    return M.lib().mgrit_cross_entropy(ctypes.byref(p) if p else None, x, y, loss, rows, grad, ws, n, None)


def test_loss_arguments():
    p = M.make_loss(B=4, V=10)
    assert _ce(None) == Bd.MGRIT_ERR_POINTER
    for bad in (dict(B=-1), dict(V=0), dict(dtype=2), dict(reduction=2), dict(reduction=-1), dict(scale=float("nan"))):
        q = M.make_loss(**dict(dict(B=4, V=10), **bad))
        assert _ce(q, n=BIG) == Bd.MGRIT_ERR_PROBLEM and M.mgrit_cross_entropy_workspace_bytes(q) == 0
    assert _ce(M.make_loss(B=1 << 30, V=1 << 10), n=BIG) == Bd.MGRIT_ERR_UNSUPPORTED
    n = M.mgrit_cross_entropy_workspace_bytes(p)
    assert n > 0 and _ce(p, n=n - 1) == Bd.MGRIT_ERR_WORKSPACE
    for k in ("x", "y", "ws"):
        assert _ce(p, n=n, **{k: None}) == Bd.MGRIT_ERR_POINTER, k
    for k in ("x", "y", "loss", "rows", "grad", "ws"):
        assert _ce(p, n=n, **{k: FAKE + 4}) == Bd.MGRIT_ERR_POINTER, k
    assert _ce(p, loss=None, rows=None, grad=None, n=n) == Bd.MGRIT_OK      # nothing wanted, nothing done


def test_clip_arguments():
    L, T = M.lib(), Bd.mgrit_tensor_t

    def call(tensors, max_norm=1.0, ws=FAKE, n=0, norm=FAKE, count=None):
        a = (T * max(1, len(tensors)))(*tensors)
        return L.mgrit_clip_gradients(a, len(tensors) if count is None else count, max_norm, norm, None, ws, n, None)

    good = T(src=FAKE, dst=FAKE, count=10, dtype=0)
    size = L.mgrit_clip_workspace_bytes((T * 1)(good), 1)
    assert size > 0 and call([good], n=size - 1) == Bd.MGRIT_ERR_WORKSPACE
    assert call([good], ws=None, n=size) == Bd.MGRIT_ERR_POINTER
    assert call([good], ws=FAKE + 8, n=size) == Bd.MGRIT_ERR_POINTER
    assert call([good], norm=FAKE + 2, n=size) == Bd.MGRIT_ERR_POINTER
    assert call([good], count=-1, n=BIG) == Bd.MGRIT_ERR_PROBLEM
    for max_norm in (-1.0, float("nan")):
        assert call([good], max_norm, n=size) == Bd.MGRIT_ERR_PROBLEM
    for bad, rc in ((T(FAKE, FAKE, -1, 0), Bd.MGRIT_ERR_PROBLEM), (T(FAKE, FAKE, 10, 2), Bd.MGRIT_ERR_PROBLEM), (T(None, FAKE, 10, 0), Bd.MGRIT_ERR_POINTER),
                    (T(FAKE + 2, FAKE, 10, 0), Bd.MGRIT_ERR_POINTER), (T(FAKE, FAKE + 1, 10, 1), Bd.MGRIT_ERR_POINTER),
                    (T(FAKE, FAKE, (1 << 40) + 1, 0), Bd.MGRIT_ERR_UNSUPPORTED)):
        assert call([good, bad], n=BIG) == rc
        assert L.mgrit_clip_workspace_bytes((T * 2)(good, bad), 2) == 0
    assert L.mgrit_clip_gradients(None, 3, 1.0, None, None, FAKE, BIG, None) == Bd.MGRIT_ERR_POINTER
    assert call([T(None, None, 0, 0)], n=0) == Bd.MGRIT_ERR_WORKSPACE         # an empty tensor's pointers are not looked at


def test_binding_refuses_tensors_that_do_not_fit():
    """What the C side cannot see: types, sizes, gaps, and tensors that are not on a GPU."""
    p = _affine()
    X, W, Y = torch.zeros(4, 8), torch.zeros(3, 8), torch.zeros(4, 3)
    call = lambda X=X, W=W, Y=Y, p=p: M.mgrit_affine_forward(p, X, W, None, None, Y, None, None)     # noqa: E731
    for kw, word in ((dict(X=X.bfloat16()), "X has type"), (dict(W=torch.zeros(3, 7)), "W has 21 values"), (dict(Y=torch.zeros(3, 4).T), "not contiguous"),
                     (dict(), "not on a GPU")):
        with pytest.raises(ValueError, match=word):
            call(**kw)
    with pytest.raises(ValueError, match="labels has type"):
        M.mgrit_cross_entropy(M.make_loss(B=4, V=3), None, torch.zeros(4, dtype=torch.int32), None, None, None, None)
    with pytest.raises(ValueError, match="has type"):
        M.make_tensor_list([torch.zeros(3, dtype=torch.float64)])
    with pytest.raises(ValueError, match="not on a GPU"):
        M.make_tensor_list([torch.zeros(3)])
    with pytest.raises(ValueError, match="1 tensors, 2 results"):
        M.make_tensor_list([X], [X, X])
    with pytest.raises(ValueError, match="no tensor given"):
        M.mgrit_clip_gradients(M.make_tensor_list([]), 1.0, None, None)


def test_overlap_rule_against_every_pair():
    """Results may lie on the tensor they replace and on nothing else; tensors that are only read may overlap."""
    import random
    r, refused = random.Random(1), 0

    def bad_pair(x, y):
        meet = x[0] < y[0] + y[1] and y[0] < x[0] + x[1]
        return meet and (x[3] or y[3]) and not (x[:3] == y[:3] and x[3] != y[3])

    for _ in range(20000):
        spans = []
        for i in range(r.randint(1, 5)):
            n, at, kind = r.randint(1, 4), r.randint(1, 30), r.random()
            spans.append((at, n, i, 0))
            if kind < 0.8:
                spans.append((at if kind < 0.4 else r.randint(1, 30), n, i, 1))
        want = any(bad_pair(x, y) for k, x in enumerate(spans) for y in spans[:k])
        try:
            Bd._refuse_overlap("x", spans)
            got = False
        except ValueError:
            got = True
        assert got == want, spans
        refused += want
    assert 2000 < refused < 18000


def test_assembly_that_writes_m0_says_so():
    """The compiler takes m0 as its own between statements unless one of them names it as an output or as overwritten."""
    csrc, found = os.path.join(ROOT, "paper_2007_07336_amd", "csrc"), 0
    for name in sorted(os.listdir(csrc)):
        if name.endswith((".hip", ".h")):
            text = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, name)).read())
            for statement in re.findall(r"\basm\s+volatile\s*\((.*?)\)\s*;", text, flags=re.S):
                if re.search(r"s_\w+\s+m0\b", statement):
                    found += 1
                    assert re.search(r'"=\{m0\}"|:\s*(?:"\w+",\s*)*"m0"', statement), (name, statement)
    assert found


def test_the_operators_take_no_memory_on_the_host():
    """The header promises that nothing is allocated, of host memory either."""
    csrc = os.path.join(ROOT, "paper_2007_07336_amd", "csrc")
    for name in ("mgrit_ops_api.hip", "mgrit_affine.hip", "mgrit_loss.hip", "mgrit_clip.hip", "mgrit_ops.h"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, name)).read())
        assert not re.search(r"\b(new|malloc|calloc|hipMalloc\w*|hipHostMalloc|std::(vector|string|map|unique_ptr|function|make_\w+))\b", text), name

"""ctypes binding of libmgrit.so.  Argument marshalling only: every step of the method runs
in the library's HIP kernels.  torch is used for device memory and the current stream.

The functions carry the names of the C entry points declared in include/mgrit.h.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmgrit.so")

MGRIT_OK = 0
MGRIT_ERR_POINTER, MGRIT_ERR_PROBLEM, MGRIT_ERR_WORKSPACE = -1, -2, -3
MGRIT_ERR_UNSUPPORTED, MGRIT_ERR_NONFINITE, MGRIT_ERR_HIP = -4, -5, -6
MGRIT_MAX_LEVELS = 16
MGRIT_INIT_ZERO, MGRIT_INIT_COPY, MGRIT_INIT_USER, MGRIT_INIT_NESTED = 0, 1, 2, 3
ERROR_NAMES = {0: "MGRIT_OK", -1: "MGRIT_ERR_POINTER", -2: "MGRIT_ERR_PROBLEM", -3: "MGRIT_ERR_WORKSPACE",
               -4: "MGRIT_ERR_UNSUPPORTED", -5: "MGRIT_ERR_NONFINITE", -6: "MGRIT_ERR_HIP"}


class MgritError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where} returned {ERROR_NAMES.get(code, code)}")
        self.code = code


class mgrit_problem_t(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("h", ctypes.c_float), ("m", ctypes.c_int32),
                ("max_levels", ctypes.c_int32), ("min_coarse", ctypes.c_int32), ("relax", ctypes.c_int32),
                ("cycle", ctypes.c_int32), ("max_iter", ctypes.c_int32), ("tol", ctypes.c_float),
                ("norm_kind", ctypes.c_int32), ("layer", ctypes.c_int32), ("act", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("B", ctypes.c_int32), ("q", ctypes.c_int32),
                ("C", ctypes.c_int32), ("Himg", ctypes.c_int32), ("Wimg", ctypes.c_int32),
                ("init", ctypes.c_int32)]


class mgrit_fc_layers_t(ctypes.Structure):
    _fields_ = [("fc_period", ctypes.c_int32), ("Wfc", ctypes.c_void_p), ("bfc", ctypes.c_void_p),
                ("dWfc", ctypes.c_void_p), ("dbfc", ctypes.c_void_p)]


class mgrit_affine_t(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int32), ("K", ctypes.c_int32), ("F", ctypes.c_int32), ("act", ctypes.c_int32),
                ("xtype", ctypes.c_int32), ("wtype", ctypes.c_int32), ("ytype", ctypes.c_int32), ("scale", ctypes.c_float)]


class mgrit_loss_t(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32), ("reduction", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class mgrit_tensor_t(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("count", ctypes.c_int64), ("dtype", ctypes.c_int32)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2007_07336_amd.build` "
                               "(or __graft_entry__.build()) first; there is no CPU fallback")
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.POINTER(mgrit_problem_t)
        vp, i32p, dp = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_double)
        L.mgrit_level_map.argtypes = [P, i32p, i32p, i32p]
        L.mgrit_level_map.restype = ctypes.c_int32
        L.mgrit_workspace_bytes.argtypes = [P]
        L.mgrit_workspace_bytes.restype = ctypes.c_size_t
        L.mgrit_adjoint_workspace_bytes.argtypes = [P]
        L.mgrit_adjoint_workspace_bytes.restype = ctypes.c_size_t
        L.mgrit_fas_forward.argtypes = [P, vp, vp, vp, vp, dp, i32p, vp, ctypes.c_size_t, vp]
        L.mgrit_fas_forward.restype = ctypes.c_int32
        L.mgrit_fas_forward_static.argtypes = [P, vp, vp, vp, vp, dp, i32p, vp]
        L.mgrit_fas_forward_static.restype = ctypes.c_int32
        L.mgrit_fas_adjoint.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, dp, i32p, vp, ctypes.c_size_t, vp]
        L.mgrit_fas_adjoint.restype = ctypes.c_int32
        L.mgrit_residual_norm.argtypes = [P, vp, vp, vp, vp, dp, vp, ctypes.c_size_t, vp]
        L.mgrit_residual_norm.restype = ctypes.c_int32
        F = ctypes.POINTER(mgrit_fc_layers_t)
        L.mgrit_workspace_bytes_mixed.argtypes = [P, ctypes.c_int32]
        L.mgrit_workspace_bytes_mixed.restype = ctypes.c_size_t
        L.mgrit_adjoint_workspace_bytes_mixed.argtypes = [P, ctypes.c_int32]
        L.mgrit_adjoint_workspace_bytes_mixed.restype = ctypes.c_size_t
        L.mgrit_fas_forward_mixed.argtypes = [P, F, vp, vp, vp, vp, dp, i32p, vp, ctypes.c_size_t, vp]
        L.mgrit_fas_forward_mixed.restype = ctypes.c_int32
        L.mgrit_fas_adjoint_mixed.argtypes = [P, F, vp, vp, vp, vp, vp, vp, vp, dp, i32p, vp, ctypes.c_size_t, vp]
        L.mgrit_fas_adjoint_mixed.restype = ctypes.c_int32
        L.mgrit_residual_norm_mixed.argtypes = [P, F, vp, vp, vp, vp, dp, vp, ctypes.c_size_t, vp]
        L.mgrit_residual_norm_mixed.restype = ctypes.c_int32
        A, X, T = ctypes.POINTER(mgrit_affine_t), ctypes.POINTER(mgrit_loss_t), ctypes.POINTER(mgrit_tensor_t)
        for name in ("mgrit_affine_workspace_bytes", "mgrit_affine_backward_workspace_bytes"):
            getattr(L, name).argtypes = [A]
            getattr(L, name).restype = ctypes.c_size_t
        L.mgrit_affine_forward.argtypes = [A, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.mgrit_affine_forward.restype = ctypes.c_int32
        L.mgrit_affine_backward.argtypes = [A, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.mgrit_affine_backward.restype = ctypes.c_int32
        L.mgrit_cross_entropy_workspace_bytes.argtypes = [X]
        L.mgrit_cross_entropy_workspace_bytes.restype = ctypes.c_size_t
        L.mgrit_cross_entropy.argtypes = [X, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.mgrit_cross_entropy.restype = ctypes.c_int32
        L.mgrit_clip_workspace_bytes.argtypes = [T, ctypes.c_int32]
        L.mgrit_clip_workspace_bytes.restype = ctypes.c_size_t
        L.mgrit_clip_gradients.argtypes = [T, ctypes.c_int32, ctypes.c_float, vp, dp, vp, ctypes.c_size_t, vp]
        L.mgrit_clip_gradients.restype = ctypes.c_int32
        L.mgrit_trace_begin.argtypes = []
        L.mgrit_trace_begin.restype = None
        L.mgrit_trace_end.argtypes = [dp, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64), dp,
                                      ctypes.c_int32]
        L.mgrit_trace_end.restype = ctypes.c_int32
        _lib = L
    return _lib


def make_problem(*, N, h, m, max_levels, relax, max_iter, layer, act, dtype, B, q=0, C=0, Himg=0, Wimg=0,
                 min_coarse=1, tol=0.0, norm_kind=0, init=1, cycle=0) -> mgrit_problem_t:
    return mgrit_problem_t(N=N, h=h, m=m, max_levels=max_levels, min_coarse=min_coarse, relax=relax, cycle=cycle,
                           max_iter=max_iter, tol=tol, norm_kind=norm_kind, layer=layer, act=act, dtype=dtype,
                           B=B, q=q, C=C, Himg=Himg, Wimg=Wimg, init=init)


def problem_from_workload(wl, **overrides) -> mgrit_problem_t:
    """Problem struct from a workload description (fields N, m, ... as in mgrit_inputs.Workload)."""
    kw = dict(N=wl.N, h=wl.h, m=wl.m, max_levels=wl.max_levels, relax=wl.relax, max_iter=wl.max_iter,
              layer=wl.layer, act=wl.act, dtype=wl.dtype, B=wl.B, q=wl.q, C=wl.C, Himg=wl.Himg, Wimg=wl.Wimg,
              min_coarse=wl.min_coarse, tol=wl.tol, norm_kind=wl.norm_kind)
    kw.update(overrides)
    return make_problem(**kw)


def mgrit_level_map(p: mgrit_problem_t):
    """Returns (N_l list, fine_index list of lists); raises MgritError on an invalid hierarchy."""
    L = lib()
    n = ctypes.c_int32(0)
    Nl = (ctypes.c_int32 * MGRIT_MAX_LEVELS)()
    rc = L.mgrit_level_map(ctypes.byref(p), ctypes.byref(n), Nl, None)
    if rc != MGRIT_OK:
        raise MgritError(rc, "mgrit_level_map")
    sizes = [Nl[i] for i in range(n.value)]
    total = sum(s + 1 for s in sizes)
    fi = (ctypes.c_int32 * total)()
    rc = L.mgrit_level_map(ctypes.byref(p), ctypes.byref(n), Nl, fi)
    if rc != MGRIT_OK:
        raise MgritError(rc, "mgrit_level_map")
    out, pos = [], 0
    for s in sizes:
        out.append([fi[pos + j] for j in range(s + 1)])
        pos += s + 1
    return sizes, out


def mgrit_workspace_bytes(p: mgrit_problem_t) -> int:
    return int(lib().mgrit_workspace_bytes(ctypes.byref(p)))


def mgrit_adjoint_workspace_bytes(p: mgrit_problem_t) -> int:
    return int(lib().mgrit_adjoint_workspace_bytes(ctypes.byref(p)))


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream or None


def mgrit_fas_forward(p: mgrit_problem_t, W, b, u0, U, workspace, *, want_hist=True, stream=None,
                      check=True):
    """Enqueues the forward solve.  Tensors are CUDA(HIP) tensors owned by the caller.
    Returns (return code, residual history list, cycles done)."""
    hist = (ctypes.c_double * max(p.max_iter, 1))() if want_hist else None
    iters = ctypes.c_int32(0)
    rc = lib().mgrit_fas_forward(ctypes.byref(p), _ptr(W), _ptr(b), _ptr(u0), _ptr(U), hist,
                                 ctypes.byref(iters) if want_hist else None, _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream))
    if check and rc != MGRIT_OK:
        raise MgritError(rc, "mgrit_fas_forward")
    return rc, ([hist[i] for i in range(iters.value)] if want_hist else None), iters.value


MGRIT_STATIC_SCRATCH_BYTES = 64 * 1024 * 1024


def mgrit_fas_forward_static(p: mgrit_problem_t, W, b, u0, U, *, want_hist=True, stream=None, check=True):
    """mgrit_fas_forward on the library's own fixed workspace (no workspace argument, nothing allocated)."""
    hist = (ctypes.c_double * max(p.max_iter, 1))() if want_hist else None
    iters = ctypes.c_int32(0)
    rc = lib().mgrit_fas_forward_static(ctypes.byref(p), _ptr(W), _ptr(b), _ptr(u0), _ptr(U), hist,
                                        ctypes.byref(iters) if want_hist else None, _stream(stream))
    if check and rc != MGRIT_OK:
        raise MgritError(rc, "mgrit_fas_forward_static")
    return rc, ([hist[i] for i in range(iters.value)] if want_hist else None), iters.value


def mgrit_fas_adjoint(p: mgrit_problem_t, W, b, U, lamN, Lam, dW, db, workspace, *, want_hist=True,
                      stream=None, check=True):
    hist = (ctypes.c_double * max(p.max_iter, 1))() if want_hist else None
    iters = ctypes.c_int32(0)
    rc = lib().mgrit_fas_adjoint(ctypes.byref(p), _ptr(W), _ptr(b), _ptr(U), _ptr(lamN), _ptr(Lam), _ptr(dW),
                                 _ptr(db), hist, ctypes.byref(iters) if want_hist else None, _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream))
    if check and rc != MGRIT_OK:
        raise MgritError(rc, "mgrit_fas_adjoint")
    return rc, ([hist[i] for i in range(iters.value)] if want_hist else None), iters.value


def mgrit_residual_norm(p: mgrit_problem_t, W, b, u0, U, workspace, *, stream=None, check=True):
    out = ctypes.c_double(0.0)
    rc = lib().mgrit_residual_norm(ctypes.byref(p), _ptr(W), _ptr(b), _ptr(u0), _ptr(U), ctypes.byref(out),
                                   _ptr(workspace), workspace.numel() * workspace.element_size(),
                                   _stream(stream))
    if check and rc != MGRIT_OK:
        raise MgritError(rc, "mgrit_residual_norm")
    return rc, out.value


def make_fc_layers(fc_period: int, Wfc, bfc, dWfc=None, dbfc=None) -> mgrit_fc_layers_t:
    """Fully connected layers of a mixed stack (device tensors owned by the caller, which keeps them alive)."""
    return mgrit_fc_layers_t(fc_period=fc_period, Wfc=_ptr(Wfc), bfc=_ptr(bfc), dWfc=_ptr(dWfc), dbfc=_ptr(dbfc))


def mgrit_workspace_bytes_mixed(p: mgrit_problem_t, fc_period: int) -> int:
    return int(lib().mgrit_workspace_bytes_mixed(ctypes.byref(p), fc_period))


def mgrit_adjoint_workspace_bytes_mixed(p: mgrit_problem_t, fc_period: int) -> int:
    return int(lib().mgrit_adjoint_workspace_bytes_mixed(ctypes.byref(p), fc_period))


def mgrit_fas_forward_mixed(p: mgrit_problem_t, fc: mgrit_fc_layers_t, W, b, u0, U, workspace, *, want_hist=True,
                            stream=None, check=True):
    hist = (ctypes.c_double * max(p.max_iter, 1))() if want_hist else None
    iters = ctypes.c_int32(0)
    rc = lib().mgrit_fas_forward_mixed(ctypes.byref(p), ctypes.byref(fc), _ptr(W), _ptr(b), _ptr(u0), _ptr(U), hist,
                                       ctypes.byref(iters) if want_hist else None, _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream))
    if check and rc != MGRIT_OK:
        raise MgritError(rc, "mgrit_fas_forward_mixed")
    return rc, ([hist[i] for i in range(iters.value)] if want_hist else None), iters.value


def mgrit_fas_adjoint_mixed(p: mgrit_problem_t, fc: mgrit_fc_layers_t, W, b, U, lamN, Lam, dW, db, workspace, *,
                            want_hist=True, stream=None, check=True):
    hist = (ctypes.c_double * max(p.max_iter, 1))() if want_hist else None
    iters = ctypes.c_int32(0)
    rc = lib().mgrit_fas_adjoint_mixed(ctypes.byref(p), ctypes.byref(fc), _ptr(W), _ptr(b), _ptr(U), _ptr(lamN),
                                       _ptr(Lam), _ptr(dW), _ptr(db), hist,
                                       ctypes.byref(iters) if want_hist else None, _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream))
    if check and rc != MGRIT_OK:
        raise MgritError(rc, "mgrit_fas_adjoint_mixed")
    return rc, ([hist[i] for i in range(iters.value)] if want_hist else None), iters.value


def mgrit_residual_norm_mixed(p: mgrit_problem_t, fc: mgrit_fc_layers_t, W, b, u0, U, workspace, *, stream=None,
                              check=True):
    out = ctypes.c_double(0.0)
    rc = lib().mgrit_residual_norm_mixed(ctypes.byref(p), ctypes.byref(fc), _ptr(W), _ptr(b), _ptr(u0), _ptr(U),
                                         ctypes.byref(out), _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream))
    if check and rc != MGRIT_OK:
        raise MgritError(rc, "mgrit_residual_norm_mixed")
    return rc, out.value


# ---- the rest of a training step: end layers, loss, clipping
MGRIT_ACT_TANH, MGRIT_ACT_RELU, MGRIT_ACT_IDENTITY = 0, 1, 2
MGRIT_FP32, MGRIT_BF16 = 0, 1
MGRIT_LOSS_SUM, MGRIT_LOSS_MEAN = 0, 1


_TYPES = []                                      # torch types by their number here, filled at the first use (torch is imported late)


def _torch_types():
    if not _TYPES:
        import torch
        _TYPES.extend((torch.float32, torch.bfloat16, torch.int64, torch.cuda, torch._C._cuda_getCurrentRawStream))
    return _TYPES


def _type(types, kind):
    return types[kind] if kind in (MGRIT_FP32, MGRIT_BF16) else None


def _check(where, items):
    """items: (name, tensor or None, number of values or None, torch type or None).  What the C side cannot see of a tensor: that it
    has this many values of this type one behind the other, on the GPU of the others.  Returns the index of that GPU, which the
    call runs on whatever the current one is; None if there is no tensor."""
    device = None
    for name, t, count, dtype in items:
        if t is None:
            continue
        d = t.get_device()
        if device is None:
            device = d
        if d < 0 or d != device or t.dtype is not dtype or (count is not None and t.numel() != count) or not t.is_contiguous():
            break
    else:
        return device
    given = [i for i in items if i[1] is not None]
    for name, t, count, dtype in given:          # something does not fit: say what
        if t.dtype is not dtype:
            raise ValueError(f"{where}: {name} has type {t.dtype}, not {dtype}")
        if count is not None and t.numel() != count:
            raise ValueError(f"{where}: {name} has {t.numel()} values, not {count}")
        if not t.is_contiguous():
            raise ValueError(f"{where}: {name} is not contiguous")
    for name, t, _, _ in given:
        if not t.is_cuda:
            raise ValueError(f"{where}: {name} is not on a GPU")
        raise_on = [n for n, u, _, _ in given if u.device != t.device]
        if raise_on:
            raise ValueError(f"{where}: {name} is on {t.device}, {raise_on[0]} is not")
    raise ValueError(f"{where}: tensors that do not fit")


def _call(where, device, stream, check, call):
    """call(stream handle) with GPU `device` the current one, on `stream` or that GPU's current stream."""
    if device is None:
        raise ValueError(f"{where}: no tensor given")
    cuda, raw_stream = _torch_types()[3:5]
    if stream is not None and stream.device_index != device:
        raise ValueError(f"{where}: the stream is on GPU {stream.device_index}, the tensors on GPU {device}")
    handle = (raw_stream(device) if stream is None else stream.cuda_stream) or None
    if cuda.current_device() == device:
        rc = call(handle)
    else:
        with cuda.device(device):
            rc = call(handle)
    if check and rc != MGRIT_OK:
        raise MgritError(rc, where)
    return rc


def _size(workspace):
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def make_affine(*, M, K, F, act=MGRIT_ACT_IDENTITY, xtype=MGRIT_FP32, wtype=MGRIT_FP32, ytype=MGRIT_FP32, scale=1.0) -> mgrit_affine_t:
    return mgrit_affine_t(M=M, K=K, F=F, act=act, xtype=xtype, wtype=wtype, ytype=ytype, scale=scale)


def mgrit_affine_workspace_bytes(p: mgrit_affine_t) -> int:
    return int(lib().mgrit_affine_workspace_bytes(ctypes.byref(p)))


def mgrit_affine_backward_workspace_bytes(p: mgrit_affine_t) -> int:
    return int(lib().mgrit_affine_backward_workspace_bytes(ctypes.byref(p)))


def _workspace(t):
    return "workspace", t, None, None if t is None else t.dtype


def mgrit_affine_forward(p: mgrit_affine_t, X, W, b, R, Y, D, workspace, *, stream=None, check=True):
    """Y = R + scale act(X W^T + b), D = scale act'(..): b, R, D may be None, and the workspace where none is needed."""
    where, T = "mgrit_affine_forward", _torch_types()
    M, K, F, y = p.M, p.K, p.F, _type(T, p.ytype)
    device = _check(where, (("X", X, M * K, _type(T, p.xtype)), ("W", W, F * K, _type(T, p.wtype)), ("b", b, F, T[0]), ("R", R, M * F, y),
                            ("Y", Y, M * F, y), ("D", D, M * F, y), _workspace(workspace)))
    return _call(where, device, stream, check, lambda s: lib().mgrit_affine_forward(
        p, _ptr(X), _ptr(W), _ptr(b), _ptr(R), _ptr(Y), _ptr(D), _ptr(workspace), _size(workspace), s))


def mgrit_affine_backward(p: mgrit_affine_t, X, W, D, dY, dX, dW, db, workspace, *, stream=None, check=True):
    """With G = dY * D (D None, identity only: scale dY): dX = G W, dW = G^T X, db = column sums of G; each may be None."""
    where, T = "mgrit_affine_backward", _torch_types()
    M, K, F, x, y = p.M, p.K, p.F, _type(T, p.xtype), _type(T, p.ytype)
    device = _check(where, (("X", X, M * K, x), ("W", W, F * K, _type(T, p.wtype)), ("D", D, M * F, y), ("dY", dY, M * F, y), ("dX", dX, M * K, x),
                            ("dW", dW, F * K, T[0]), ("db", db, F, T[0]), _workspace(workspace)))
    return _call(where, device, stream, check, lambda s: lib().mgrit_affine_backward(
        p, _ptr(X), _ptr(W), _ptr(D), _ptr(dY), _ptr(dX), _ptr(dW), _ptr(db), _ptr(workspace), _size(workspace), s))


def make_loss(*, B, V, dtype=MGRIT_FP32, reduction=MGRIT_LOSS_MEAN, scale=1.0) -> mgrit_loss_t:
    return mgrit_loss_t(B=B, V=V, dtype=dtype, reduction=reduction, scale=scale)


def mgrit_cross_entropy_workspace_bytes(p: mgrit_loss_t) -> int:
    return int(lib().mgrit_cross_entropy_workspace_bytes(ctypes.byref(p)))


def mgrit_cross_entropy(p: mgrit_loss_t, logits, labels, loss, row_loss, grad, workspace, *, stream=None, check=True):
    """loss (1 value), row_loss (B) and grad (like logits, may be logits) may each be None; labels are int64."""
    where, T = "mgrit_cross_entropy", _torch_types()
    t, B, V = _type(T, p.dtype), p.B, p.V
    device = _check(where, (("logits", logits, B * V, t), ("labels", labels, B, T[2]), ("loss", loss, 1, T[0]), ("row_loss", row_loss, B, T[0]),
                            ("grad", grad, B * V, t), _workspace(workspace)))
    return _call(where, device, stream, check, lambda s: lib().mgrit_cross_entropy(
        p, _ptr(logits), _ptr(labels), _ptr(loss), _ptr(row_loss), _ptr(grad), _ptr(workspace), _size(workspace), s))


def _refuse_overlap(where, spans):
    """Refuses results that overlap a tensor other than the one they replace, or another result: a tensor that is listed twice would
    be scaled twice.  spans: (address, bytes, index, 1 for a result)."""
    furthest = [[(0, -1), (0, -1)], [(0, -1), (0, -1)]]       # of all spans and of results: the two furthest ends of different indices
    place = {}
    for at, size, i, k in sorted(spans):
        others = furthest[0 if k else 1]
        end = others[0][0] if others[0][1] != i else others[1][0]
        mine = place.setdefault(i, (at, size))
        if at < end or (mine != (at, size) and at < mine[0] + mine[1]):
            raise ValueError(f"{where}: {'result' if k else 'tensor'} {i} overlaps another one")
        for f in furthest[:2 if k else 1]:
            if i == f[0][1]:
                f[0] = (max(f[0][0], at + size), i)
            elif at + size > f[0][0]:
                f[0], f[1] = (at + size, i), f[0]
            elif i == f[1][1] or at + size > f[1][0]:
                f[1] = (max(at + size, f[1][0] if i == f[1][1] else 0), i)


class TensorList:
    """Tensors to clip: the descriptors handed to the library, and the tensors, which are kept alive."""

    def __init__(self, src: Sequence, dst: Optional[Sequence] = None):
        where, dst, T = "make_tensor_list", list(src) if dst is None else list(dst), _torch_types()
        self.src, self.dst = list(src), dst
        if len(self.src) != len(self.dst):
            raise ValueError(f"{where}: {len(self.src)} tensors, {len(self.dst)} results")
        self.array = (mgrit_tensor_t * max(1, len(self.src)))()
        self.device, spans = None, []
        for i, (a, b) in enumerate(zip(self.src, self.dst)):
            if a.dtype not in T[:2]:
                raise ValueError(f"{where}: tensor {i} has type {a.dtype}")
            device = _check(where, ((f"tensor {i}", a, None, a.dtype), (f"result {i}", b, a.numel(), a.dtype)))
            if self.device is not None and device != self.device:
                raise ValueError(f"{where}: tensor {i} is on GPU {device}, others on GPU {self.device}")
            self.device = device
            spans += [(t.data_ptr(), t.numel() * t.element_size(), i, k) for k, t in enumerate((a, b)) if t is not None and t.numel()]
            self.array[i] = mgrit_tensor_t(src=_ptr(a), dst=_ptr(b), count=a.numel(), dtype=T.index(a.dtype))

        _refuse_overlap(where, spans)

    def __len__(self):
        return len(self.src)


def make_tensor_list(src: Sequence, dst: Optional[Sequence] = None) -> TensorList:
    """Tensors and where their clipped values go (None: into themselves; a None among dst: that tensor only counts)."""
    return TensorList(src, dst)


def mgrit_clip_workspace_bytes(tensors: TensorList) -> int:
    return int(lib().mgrit_clip_workspace_bytes(tensors.array, len(tensors)))


def mgrit_clip_gradients(tensors: TensorList, max_norm: float, norm, workspace, *, want_norm=False, stream=None, check=True):
    """dst = src * min(1, max_norm / norm).  norm: one float on the GPU or None.  Returns (return code, the norm if want_norm, which
    waits for the GPU)."""
    where, host, T = "mgrit_clip_gradients", ctypes.c_double(0.0) if want_norm else None, _torch_types()
    device = _check(where, (("norm", norm, 1, T[0]), _workspace(workspace)))
    if device is None:
        device = tensors.device
    elif tensors.device is not None and device != tensors.device:
        raise ValueError(f"{where}: norm or workspace on GPU {device}, the tensors on GPU {tensors.device}")
    rc = _call(where, device, stream, check, lambda s: lib().mgrit_clip_gradients(
        tensors.array, len(tensors), max_norm, _ptr(norm), None if host is None else ctypes.byref(host), _ptr(workspace), _size(workspace), s))
    return rc, None if host is None else host.value


TRACE_CLASSES = ("dense_step_kernel<float,64,64>", "dense_step_kernel<float,128,128>",
                 "dense_step_kernel<bf16,64,64>", "dense_step_kernel<bf16,128,128>",
                 "conv_step_kernel<float>", "conv_step_kernel<bf16>", "dense_grad_kernel",
                 "dense_sweep_kernel<float>", "dense_sweep_kernel<bf16>", "dense_ksplit_kernel<float,8>",
                 "dense_ksplit_kernel<float,4>", "dense_ksplit_kernel<bf16,4>", "dense_ksplit_kernel<bf16,8>",
                 "conv_sweep_kernel")


def mgrit_trace_begin() -> None:
    lib().mgrit_trace_begin()


def mgrit_trace_end() -> dict:
    """{kernel class: (total ms, launches, layer steps, algorithmic bytes)} of the launches since
    mgrit_trace_begin()."""
    n = len(TRACE_CLASSES)
    ms = (ctypes.c_double * n)()
    la = (ctypes.c_int64 * n)()
    un = (ctypes.c_int64 * n)()
    by = (ctypes.c_double * n)()
    rc = lib().mgrit_trace_end(ms, la, un, by, n)
    if rc != MGRIT_OK:
        raise MgritError(rc, "mgrit_trace_end")
    return {TRACE_CLASSES[i]: (ms[i], la[i], un[i], by[i]) for i in range(n) if la[i] > 0}

"""Norms after and before a block with its gate and residual step, forwards and backwards, against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2007_07336_amd as M
from tests.ops_util import HALF, KIND, TINY, TYPES, near, normal

pytestmark = pytest.mark.gpu
NAN = float("nan")
GATE = {"none": M.MGRIT_GATE_NONE, "feature": M.MGRIT_GATE_FEATURE, "entry": M.MGRIT_GATE_ENTRY}
KIND_OF = {"rms": M.MGRIT_NORM_ROOT, "layer": M.MGRIT_NORM_LAYER}


def norm_of(x, kind, eps):
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    d = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + eps)
    return x * d, d


class Block:
    def __init__(self, rows, q, kind="rms", gate="none", types="ff", post=True, pre=True, eps=1.0e-5, scale=0.7, seed=0, wide=1.0):
        self.rows, self.q, self.kind, self.types, self.eps, self.scale = rows, q, kind, types, eps, scale
        st, ft = types
        self.p = M.make_block_norm(M=rows, q=q, kind=KIND_OF[kind], gate=GATE[gate], stype=KIND[st], ftype=KIND[ft], eps=eps, scale=scale)
        self.f, self.r = normal((rows, q), wide, ft, seed + 1), normal((rows, q), 1.0, st, seed + 2)
        self.gate = {"none": None, "feature": normal((q,), 0.5, "f", seed + 3), "entry": normal((rows, q), 0.5, ft, seed + 3)}[gate]
        self.post = 1.0 + normal((q,), 0.2, "f", seed + 4) if post else None
        self.pre = 1.0 + normal((q,), 0.2, "f", seed + 5) if pre else None
        self.dS, self.dY = normal((rows, q), 1.0, st, seed + 6), normal((rows, q), 1.0, ft, seed + 7) if pre else None
        n = M.mgrit_block_norm_workspace_bytes(self.p)
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")

    def new(self, t, *shape):
        return torch.full(shape, NAN, dtype=TYPES[t], device="cuda")

    def forward(self, **kw):
        st, ft = self.types
        S, Y = self.new(st, self.rows, self.q), self.new(ft, self.rows, self.q) if self.pre is not None else None
        M.mgrit_block_norm_forward(self.p, self.f, self.r, self.gate, self.post, self.pre, S, Y, **kw)
        return S, Y

    def backward(self, S, dS="own", **kw):
        st, ft = self.types
        shape = (self.rows, self.q)
        o = dict(df=self.new(ft, *shape), dr=self.new(st, *shape), dgate=None if self.gate is None else torch.full_like(self.gate, NAN),
                 dpost=None if self.post is None else self.new("f", self.q), dpre=None if self.pre is None else self.new("f", self.q))
        M.mgrit_block_norm_backward(self.p, self.f, S, self.gate, self.post, self.pre, self.dS if dS == "own" else dS, self.dY, o["df"], o["dr"], o["dgate"],
                                    o["dpost"], o["dpre"], self.ws, **kw)
        return o

    # One step is 2^-23 of a sum's magnitudes for each of its additions and a few more for the operations around it.  A sum over q is formed by
    # threads of at most ceil(q / 512) + 8 .. entries and a tree; q steps bound it in any order.
    def steps(self):
        return (self.q + 24) * 2.0 ** -23

    def check_forward(self):
        S, Y = self.forward()
        d = {k: None if v is None else v.double() for k, v in dict(f=self.f, r=self.r, gate=self.gate, post=self.post, pre=self.pre).items()}
        e = self.steps()
        n, nb = d["f"], 0.0
        if d["post"] is not None:
            x, dev = norm_of(d["f"], self.kind, self.eps)
            # the mean is e of the mean magnitude off, the deviation e / 2 relative (its sum has positive terms) plus what the mean's error makes of it
            off = e * d["f"].abs().mean(1, keepdim=True) if self.kind == "layer" else 0.0
            n, nb = x * d["post"], (e * x.abs() + off * dev * (1.0 + x.abs())) * d["post"].abs()
        g = 1.0 if d["gate"] is None else d["gate"]
        want = d["r"] + self.scale * g * n
        sb = 2.0 ** -21 * (want.abs() + abs(self.scale) * (n * g).abs()) + abs(self.scale) * (g.abs() if torch.is_tensor(g) else 1.0) * nb
        near(S, want, sb, ("S", self.rows, self.q, self.kind, self.types))
        if d["pre"] is not None:
            y, dev = norm_of(want, self.kind, self.eps)
            top = sb.pow(2).mean(1, keepdim=True).sqrt()                    # the errors' part in the mean and the deviation
            off = (e * want.abs().mean(1, keepdim=True) + top) if self.kind == "layer" else 0.0
            yb = (e * y.abs() + dev * (sb + top * y.abs() + off * (1.0 + y.abs()))) * d["pre"].abs()
            near(Y, y * d["pre"], yb, ("Y", self.rows, self.q, self.kind, self.types))
        return S, Y

    def exact_backward(self, S, dS):
        """Gradients in 64 bits, and what floats may be off them (each the magnitudes of what it is put together from)."""
        d = {k: None if v is None else v.double() for k, v in dict(f=self.f, S=S, gate=self.gate, post=self.post, pre=self.pre, dS=dS, dY=self.dY).items()}
        layer, a, e = self.kind == "layer", self.scale, self.steps()
        mean = lambda t: t.mean(1, keepdim=True)                                                       # noqa: E731
        ds = d["dS"] if dS is not None else torch.zeros_like(d["f"])
        mag, want, bound = ds.abs(), {}, {}
        if d["pre"] is not None:
            sn, dev = norm_of(d["S"], self.kind, self.eps)
            h = d["dY"] * d["pre"]
            ds = ds + dev * (h - sn * mean(h * sn) - (mean(h) if layer else 0.0))
            off = 1.0 + mean(d["S"].abs()) * dev if layer else 1.0           # (the mean's error, in units of x^)
            mag = mag + dev * (h.abs() + (sn.abs() + off) * mean(h.abs() * (sn.abs() + off)) * (1.0 + sn.abs()) + mean(h.abs()))
            want["dpre"], bound["dpre"] = (d["dY"] * sn).sum(0), (d["dY"].abs() * (sn.abs() + off)).sum(0)
        want["dr"], bound["dr"] = ds, mag
        g = torch.ones_like(ds) if d["gate"] is None else d["gate"].expand_as(ds)
        t, tm = a * ds, abs(a) * mag
        fn, fm, w = d["f"], d["f"].abs(), 1.0
        if d["post"] is not None:
            fn, fdev = norm_of(d["f"], self.kind, self.eps)
            foff = 1.0 + mean(d["f"].abs()) * fdev if layer else 1.0
            fm, w = fn.abs() + foff, d["post"]
        dn, dm = t * g, tm * g.abs()
        if d["gate"] is not None:
            want["dgate"], bound["dgate"] = t * fn * w, tm * fm * (w.abs() if torch.is_tensor(w) else 1.0)
            if d["gate"].dim() == 1:
                want["dgate"], bound["dgate"] = want["dgate"].sum(0), bound["dgate"].sum(0)
        if d["post"] is not None:
            want["dpost"], bound["dpost"] = (dn * fn).sum(0), (dm * fm).sum(0)
            dn, dm = dn * w, dm * w.abs()
            dn = fdev * (dn - fn * mean(dn * fn) - (mean(dn) if layer else 0.0))
            dm = fdev * (dm + fm * mean(dm * fm) * (1.0 + fn.abs()) + mean(dm))
        want["df"], bound["df"] = dn, dm
        return want, {k: (2.0 * e + (self.rows + 8) * 2.0 ** -23 * (v.dim() == 1)) * v + TINY for k, v in bound.items()}

    def check_backward(self, S, dS="own"):
        got = self.backward(S, dS)
        want, bound = self.exact_backward(S, self.dS if dS == "own" else dS)
        for k, w in want.items():
            near(got[k], w, bound[k], (k, self.rows, self.q, self.kind, self.types))
        return got


SIZES = [(1, 1), (3, 8), (5, 7), (2, 64), (9, 511), (4, 513), (6, 1031), (3, 2048), (3, 2056), (2, 4100), (2, 8191), (2, 8200), (2, 16391)]


@pytest.mark.parametrize("rows,q", SIZES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_sizes(rows, q, kind):
    b = Block(rows, q, kind, "feature" if q % 2 else "entry", "ff", seed=q)
    S, _ = b.check_forward()
    b.check_backward(S)


@pytest.mark.parametrize("types", ["ff", "fb", "bf", "bb"])
@pytest.mark.parametrize("gate", ["none", "feature", "entry"])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (True, False), (False, False)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_forms(types, gate, post, pre, kind):
    for rows, q in ((7, 130), (3, 1000), (2, 9001)):
        b = Block(rows, q, kind, gate, types, post, pre, seed=q)
        S, _ = b.check_forward()
        b.check_backward(S)
        b.check_backward(S, None)


@pytest.mark.parametrize("rows", [511, 600, 5000, 20000])
def test_many_rows(rows):
    b = Block(rows, 72, "layer", "feature", "fb", seed=rows)
    S, _ = b.check_forward()
    b.check_backward(S)


def test_against_differences():
    """The gradients of <S, dS> + <Y, dY> against central differences of the forward pass in 64 bits."""
    b = Block(3, 24, "layer", "feature", "ff", eps=1.0e-2, seed=5)
    leaves = {k: getattr(b, k).double() for k in ("f", "r", "gate", "post", "pre")}

    def value(v):
        S = v["r"] + b.scale * v["gate"] * norm_of(v["f"], b.kind, b.eps)[0] * v["post"]
        return float((S * b.dS.double()).sum() + (norm_of(S, b.kind, b.eps)[0] * v["pre"] * b.dY.double()).sum())

    S, _ = b.forward()
    got = b.backward(S)
    for name, grad in (("f", "df"), ("r", "dr"), ("gate", "dgate"), ("post", "dpost"), ("pre", "dpre")):
        flat = leaves[name].reshape(-1)
        for i in range(0, flat.numel(), 5):
            step, old = 1.0e-5, float(flat[i])
            flat[i] = old + step
            up = value(leaves)
            flat[i] = old - step
            down = value(leaves)
            flat[i] = old
            d = (up - down) / (2 * step)
            # third derivatives times step^2 (values of a few units over deviations of one: 1e3 at most) and 1e-14 / step of rounding in 64 bits;
            # the float result, and S as it was stored, 24 bits of sums of 24 terms of a few units
            assert abs(float(got[grad].reshape(-1)[i]) - d) <= 1.0e3 * step ** 2 + 1.0e-8 + 200 * 2.0 ** -24 * max(1.0, abs(d)), (name, i)


def test_in_place_and_outputs_that_are_not_wanted():
    b = Block(5, 1500, "layer", "entry", "ff", seed=3)
    S, Y = b.forward()
    want = b.backward(S)
    f, r = b.f.clone(), b.r.clone()
    M.mgrit_block_norm_forward(b.p, f, r, b.gate, b.post, b.pre, r, f)             # S in r's place, Y in f's
    assert torch.equal(r, S) and torch.equal(f, Y)
    for q in (1500, 17000):
        b = Block(3, q, "layer", "entry", "ff", seed=3)
        S, _ = b.forward()
        want = b.backward(S)
        dS, dY, f = b.dS.clone(), b.dY.clone(), b.f.clone()
        M.mgrit_block_norm_backward(b.p, b.f, S, b.gate, b.post, b.pre, dS, dY, dY, dS, None, None, None, b.ws)
        assert torch.equal(dS, want["dr"]) and torch.equal(dY, want["df"])
        M.mgrit_block_norm_backward(b.p, f, S, b.gate, b.post, b.pre, b.dS, b.dY, f, None, None, None, None, b.ws)
        assert torch.equal(f, want["df"])
        o = torch.full((q,), NAN, device="cuda")
        M.mgrit_block_norm_backward(b.p, b.f, S, b.gate, b.post, b.pre, b.dS, b.dY, None, None, None, o, None, b.ws)
        assert torch.equal(o, want["dpost"])


@pytest.mark.parametrize("q", [40, 100, 200, 6000, 12000, 17000])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_forward_in_place_in_each_form(kind, q):
    """S in r's place and Y in f's where several rows share a wavefront, where a row takes two vectors a thread and where it is read for every step."""
    b = Block(5, q, kind, "feature", "ff", seed=q)
    S, Y = b.forward()
    f, r = b.f.clone(), b.r.clone()
    M.mgrit_block_norm_forward(b.p, f, r, b.gate, b.post, b.pre, r, f)
    assert torch.equal(r, S) and torch.equal(f, Y)


def test_no_rows_and_rows_that_are_not_finite():
    b = Block(0, 40, gate="feature")
    b.forward()
    o = b.backward(b.r)
    assert all(bool((o[k] == 0).all()) for k in ("dgate", "dpost", "dpre"))
    b = Block(4, 300, "layer", "none", "fb", seed=9)
    S0, Y0 = b.forward()
    b.f[1, 5], b.f[2, 7] = NAN, math.inf
    S, Y = b.forward()
    for t, t0 in ((S, S0), (Y, Y0)):                                              # they stay in their rows
        assert torch.equal(t[[0, 3]], t0[[0, 3]]) and bool(torch.isnan(t[1:3]).all())
    o = b.backward(S)
    assert not bool(torch.isnan(o["df"][[0, 3]]).any()) and bool(torch.isnan(o["df"][1:3]).all()) and bool(torch.isnan(o["dpre"]).all())
    z = Block(2, 64, "rms", "none", "ff", eps=0.0)
    z.f.zero_()
    S, Y = z.forward()
    assert bool(torch.isnan(S).all())
    # rows of very large entries: their squares stay finite below 1e19, and small ones keep their digits beside eps
    w = Block(2, 200, "rms", "none", "ff", eps=1.0e-30, seed=4, wide=1.0e-12)
    w.check_forward()


def test_replays_beside_eager_work():
    b = Block(70, 700, "layer", "feature", "fb", seed=8)
    S, _ = b.forward()
    out = b.backward(S)
    names = [k for k in out if out[k] is not None]
    run = lambda: M.mgrit_block_norm_backward(b.p, b.f, S, b.gate, b.post, b.pre, b.dS, b.dY, out["df"], out["dr"], out["dgate"], out["dpost"], out["dpre"],   # noqa: E731
                                              b.ws)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        run()
    for replay in range(3):
        b.dY.copy_(normal(b.dY.shape, 1.0, "b", 50 + replay))
        run()
        want = {k: out[k].clone() for k in names}
        for k in names:
            out[k].fill_(NAN)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[k]) for k in names), replay

"""Arrays in few bits: packing against the definition, bit for bit; products with packed weights and backward passes from kept activations
against the same values in 64 bits."""
import math

import pytest
import torch

import paper_2007_07336_amd as M
from tests.ops_util import ACT, KIND, TYPES, Affine, near, normal, sum_bound

pytestmark = pytest.mark.gpu
FORMAT = {"mx8": M.MGRIT_MX8, "mx4": M.MGRIT_MX4}
GRID4 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
GRID8 = torch.tensor([(m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127], dtype=torch.float64)


def values_of(x, form):
    """The packed values of a float or bf16 array, by the definition, in double on the CPU."""
    x = x.detach().cpu().double()
    rows, cols = x.shape
    grid = GRID4 if form == "mx4" else GRID8
    pad = torch.zeros((rows, (cols + 31) // 32 * 32), dtype=torch.float64)
    pad[:, :cols] = x
    blocks = pad.view(-1, 32)
    out = torch.empty_like(blocks)
    top = blocks.abs().max(1).values
    largest = float(grid[-1])
    for b in range(blocks.shape[0]):
        t = float(top[b])
        if not math.isfinite(t):
            out[b] = math.nan
            continue
        s = -127
        while t > largest * 2.0 ** s:
            s += 1
        v = blocks[b].abs() * 2.0 ** -s
        hi = torch.searchsorted(grid, v).clamp(max=len(grid) - 1)
        lo = (hi - 1).clamp(min=0)
        up = (v - grid[lo] > grid[hi] - v) | ((v - grid[lo] == grid[hi] - v) & (hi % 2 == 0))
        out[b] = torch.where(up, grid[hi], grid[lo]) * torch.sign(blocks[b]) * 2.0 ** s
    return out.view(rows, -1)[:, :cols]


def packed(x, form):
    p = M.make_packed(rows=x.shape[0], cols=x.shape[1], format=FORMAT[form], dtype=KIND["b" if x.dtype == torch.bfloat16 else "f"])
    n = M.mgrit_packed_bytes(p)
    room = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    M.mgrit_pack(p, x, room[:n])
    assert bool((room[n:] == 0xA5).all())
    return p, room[:n]


def unpacked(p, a, t):
    q = M.make_packed(rows=p.rows, cols=p.cols, format=p.format, dtype=KIND[t])
    out = torch.full((p.rows, p.cols), 7.0, dtype=TYPES[t], device="cuda")
    M.mgrit_unpack(q, a, out)
    return out


@pytest.mark.parametrize("form", ["mx8", "mx4"])
@pytest.mark.parametrize("t", ["f", "b"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 33), (2, 256), (5, 257), (4, 1031), (33, 520), (2, 4096)])
def test_values(form, t, rows, cols):
    x = normal((rows, cols), 1.0, t, rows + cols)
    x.mul_(torch.exp(normal((rows, 1), 3.0, "f", 1)).to(x.dtype))
    p, a = packed(x, form)
    want = values_of(x, form)
    assert torch.equal(unpacked(p, a, "f").cpu().double(), want)
    assert torch.equal(unpacked(p, a, "b").cpu().double(), want)              # (7 or 4 bits and a power of two in its range)


@pytest.mark.parametrize("form", ["mx8", "mx4"])
def test_every_bf16_value_and_ties(form):
    """All finite bf16 values beside a block's largest one of several magnitudes, and floats a step off the ties."""
    bits = torch.arange(0, 1 << 16, dtype=torch.int32)
    x = (bits << 16).view(torch.float32)
    x = x[torch.isfinite(x)]
    x = torch.nn.functional.pad(x, (0, -len(x) % 31)).view(-1, 31)
    lead = torch.cat([torch.full((x.shape[0], 1), v) for v in (1.0, 447.9, 448.0, 448.1, 6.0, 6.001, 7.5, 1.0e-38, 3.0e38)], 0)
    x = torch.cat([lead, x.repeat(9, 1)], 1)[::7].contiguous()
    for y in (x, torch.nextafter(x, torch.zeros_like(x)), torch.nextafter(x, torch.full_like(x, 3.4e38)).clamp(-3.3e38, 3.3e38)):
        p, a = packed(y.cuda(), form)
        # (as floats: the largest ones round up to 2^128, which is none)
        got, want = unpacked(p, a, "f").cpu(), values_of(y, form).float()
        assert torch.equal(got, want), (got - want).abs().max()


@pytest.mark.parametrize("form", ["mx8", "mx4"])
def test_ends_of_the_range(form):
    x = torch.zeros((8, 96), device="cuda")
    x[1, 3] = 2.0 ** -149
    x[2, 3], x[2, 40] = 2.0 ** -127, -3.0e-39
    x[3, 3], x[3, 40], x[3, 41] = torch.finfo(torch.float32).max, torch.finfo(torch.float32).min, 1.0
    x[4, 33] = math.inf
    x[5, 33], x[5, 2] = math.nan, -0.0
    x[6, 95] = -math.inf
    x[7, :] = torch.arange(96, device="cuda") * 2.0 ** -140
    p, a = packed(x, form)
    got, want = unpacked(p, a, "f").cpu(), values_of(x.cpu(), form).float()          # (the largest floats round up to 2^128, which is none)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and bool(torch.isnan(got[4, 32:64]).all()) and not bool(torch.isnan(got[4, :32]).any())
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def test_layout():
    """The array as the header describes it: codes, then scales by slabs."""
    x = normal((3, 300), 1.0, "f", 1)
    for form, code in (("mx8", 512), ("mx4", 256)):
        p, a = packed(x, form)
        codes, at = a[:3 * code].view(3, code).cpu(), (3 * code + 255) // 256 * 256
        scales = a[at:at + 2 * 3 * 8].view(2, 3, 8).cpu().double()
        want = values_of(x, form)
        for r in range(3):
            for k in (0, 1, 31, 32, 64, 100, 255, 256, 290, 299):
                block = k // 32
                s = scales[block // 8, r, (block % 2) * 4 + block % 8 // 2] - 127
                c = int(codes[r, k]) if form == "mx8" else int(codes[r, k // 2]) >> 4 * (k % 2) & 15
                top, grid = (128, GRID8) if form == "mx8" else (8, GRID4)
                assert float(grid[c % top]) * (-1 if c >= top else 1) * 2.0 ** float(s) == float(want[r, k]), (form, r, k)
        assert bool((codes[:, 300 * code // 512:] == 0).all())


class PackedLayer:
    def __init__(self, rows, K, F, x="b", form="bf16", y="b", act="identity", scale=1.0, bias=True, residual=False, seed=0):
        self.what = (rows, K, F, x, form, y, act)
        self.p = M.make_affine_packed(M=rows, K=K, F=F, act=ACT[act], xtype=KIND[x], xformat=M.MGRIT_MX4 if form == "mx4" else M.MGRIT_BF16, ytype=KIND[y],
                                      scale=scale)
        self.rows, self.K, self.F, self.y, self.act, self.scale = rows, K, F, y, act, scale
        self.X, W = normal((rows, K), 1.0, x, seed + 1), normal((F, K), K ** -0.5, "b", seed + 2)
        w, self.W = packed(W, "mx4")
        self.b = normal((F,), 0.3, "f", seed + 3) if bias else None
        self.R = normal((rows, F), 1.0, y, seed + 4) if residual else None
        self.Wv = unpacked(w, self.W, "f").double()
        n = M.mgrit_affine_packed_workspace_bytes(self.p)
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        if form == "mx4":
            q, a = packed(self.X, "mx4")
            self.Xv = unpacked(q, a, "f").double()
        else:
            self.Xv = self.X.bfloat16().double()

    def run(self, factor=False, **kw):
        Y = torch.full((self.rows, self.F), float("nan"), dtype=TYPES[self.y], device="cuda")
        D = torch.full_like(Y, float("nan")) if factor else None
        M.mgrit_affine_packed_forward(self.p, self.X, self.W, self.b, self.R, Y, D, self.ws, **kw)
        return Y, D

    def check(self, factor=False):
        Y, D = self.run(factor)
        z, zb = self.Xv @ self.Wv.T, sum_bound(self.Xv, self.Wv, self.K)
        if self.b is not None:
            z = z + self.b.double()
            zb = zb + 2.0 ** -23 * z.abs()
        s = self.scale
        if self.act == "tanh":                       # (slopes and the function's own error: see tests/ops_util.py)
            y, d = torch.tanh(z), 1.0 / torch.cosh(z) ** 2
            yb, db = zb + 2.0 ** -21 * y.abs(), zb + 2.0 ** -20 * d
        elif self.act == "relu":
            y, d, yb, db = torch.relu(z), (z > 0).double(), zb, (z.abs() <= zb).double()
        else:
            y, d, yb, db = z, torch.ones_like(z), zb, torch.zeros_like(z)
        r = self.R.double() if self.R is not None else torch.zeros_like(z)
        near(Y, r + s * y, abs(s) * (yb + 2.0 ** -23 * y.abs()), ("Y",) + self.what)
        if factor:
            near(D, s * d, abs(s) * (db + 2.0 ** -23 * d), ("D",) + self.what)
        return Y


SIZES = [(1, 1, 1), (1, 31, 5), (1, 4096, 130), (2, 257, 64), (16, 256, 65), (17, 1000, 33), (33, 640, 513), (64, 512, 96), (65, 300, 70), (100, 1031, 517),
         (130, 8, 200), (300, 256, 300), (257, 2049, 260), (5, 70, 1200), (48, 4096, 300)]


@pytest.mark.parametrize("rows,K,F", SIZES)
@pytest.mark.parametrize("form", ["bf16", "mx4"])
@pytest.mark.parametrize("x", ["f", "b"])
def test_products(rows, K, F, form, x):
    PackedLayer(rows, K, F, x, form, "f" if rows % 2 else "b", "tanh" if F % 2 else "identity", 0.5, residual=K % 2 == 0, bias=F % 3 > 0, seed=rows).check()


@pytest.mark.parametrize("form", ["bf16", "mx4"])
@pytest.mark.parametrize("act", ["tanh", "relu", "identity"])
@pytest.mark.parametrize("y", ["f", "b"])
def test_epilogues(form, act, y):
    for rows, K, F in ((7, 264, 100), (90, 264, 100), (600, 512, 520), (1100, 300, 1030)):
        PackedLayer(rows, K, F, "b", form, y, act, -0.25, residual=True, seed=F).check(factor=True)


@pytest.mark.parametrize("form", ["bf16", "mx4"])
def test_large_products(form):
    """Tiles of 256, with whole and with ragged edges."""
    PackedLayer(2048, 1024, 4096, "b", form, "b", "tanh", 0.5, residual=True, seed=1).check(factor=True)
    PackedLayer(4100, 770, 2050, "f", form, "f", "relu", 1.0, seed=2).check()


@pytest.mark.parametrize("form", ["bf16", "mx4"])
@pytest.mark.parametrize("rows", [3, 70, 600])
def test_values_that_are_not_finite_stay_in_their_rows(form, rows):
    a = PackedLayer(rows, 300, 80, "f", form, "f", seed=rows)
    want, _ = a.run()
    a.X[1, 299], a.X[rows - 1, 0] = math.nan, math.inf
    got, _ = a.run()
    keep = torch.ones(rows, dtype=torch.bool)
    keep[[1, rows - 1]] = False
    assert torch.equal(got[keep], want[keep]) and bool(torch.isnan(got[1]).all()) and not bool(torch.isfinite(got[rows - 1]).any())


def test_no_rows_streams_and_replays():
    z = M.make_affine_packed(M=0, K=10, F=3)
    w = torch.zeros(M.mgrit_packed_bytes(M.make_packed(rows=3, cols=10, format=M.MGRIT_MX4)), dtype=torch.uint8, device="cuda")
    e = torch.zeros((0, 3), device="cuda")
    M.mgrit_affine_packed_forward(z, torch.zeros((0, 10), device="cuda"), w, None, None, e, None, None)
    for form, rows in (("bf16", 5), ("mx4", 5), ("bf16", 200), ("mx4", 700)):
        a = PackedLayer(rows, 520, 300, "f", form, "f", seed=4)
        Y, _ = a.run()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        Z, _ = a.run(stream=side)
        side.synchronize()
        out = torch.zeros_like(Y)
        go = lambda: M.mgrit_affine_packed_forward(a.p, a.X, a.W, a.b, a.R, out, None, a.ws)         # noqa: E731
        graph = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            go()
        for replay in range(3):
            a.X.copy_(normal(a.X.shape, 1.0, "f", 60 + replay))
            go()
            want = out.clone()
            out.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), (form, rows, replay)


# ---------------------------------------------------------------------------------------------- kept activations
def kept(rows, K, F, types, act, seed=0):
    """An affine layer whose inputs and factors are those that come back from 8 bits, and the packed arrays."""
    a = Affine(rows, K, F, types, act, 0.5 if act != "identity" else 0.75, seed=seed)
    D = None if act == "identity" else (0.5 * torch.rand((rows, F), generator=torch.Generator().manual_seed(seed + 9))).to(TYPES[types[2]]).cuda()
    px, X8 = packed(a.X, "mx8")
    D8 = None
    if D is not None:
        pd, D8 = packed(D, "mx8")
        D = unpacked(pd, D8, "f")
    return a, unpacked(px, X8, "f"), X8, D, D8


def run_kept(a, X8, D8, **kw):
    n = M.mgrit_affine_kept_workspace_bytes(a.p)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None
    dX, dW, db = a.new((a.rows, a.K), a.types[0]), a.new((a.F, a.K)), a.new((a.F,))
    M.mgrit_affine_kept_backward(a.p, X8, a.W, D8, a.dY, dX, dW, db, ws, **kw)
    return dX, dW, db


@pytest.mark.parametrize("types", ["fff", "bbb", "fbf", "ffb", "bbf"])
@pytest.mark.parametrize("act", ["tanh", "relu", "identity"])
@pytest.mark.parametrize("rows,K,F", [(1, 1, 1), (3, 300, 10), (40, 33, 70), (33, 2000, 9), (300, 257, 16), (130, 520, 260), (520, 1031, 70), (600, 512, 640)])
def test_backward_from_kept_activations(types, act, rows, K, F):
    a, X, X8, D, D8 = kept(rows, K, F, types, act, rows)
    dX, dW, db = run_kept(a, X8, D8)
    G = a.dY.double() * (D.double() if D is not None else a.scale)
    what, W = (rows, K, F, types, act), a.W.double()
    near(dX, G @ W, sum_bound(G, W.T, F + 2), ("dX",) + what)
    near(dW, G.T @ X.double(), sum_bound(G.T, X.double().T, rows + 2), ("dW",) + what)
    near(db, G.sum(0), (rows + 4) * 2.0 ** -23 * G.abs().sum(0) + rows * 2.0 ** -126, ("db",) + what)


def test_backward_from_kept_activations_of_a_large_layer():
    a, X, X8, D, D8 = kept(2048, 1024, 2048, "bbb", "tanh", 3)
    dX, dW, db = run_kept(a, X8, D8)
    G, W = a.dY.double() * D.double(), a.W.double()
    near(dX, G @ W, sum_bound(G, W.T, 2050), "dX")
    near(dW, G.T @ X.double(), sum_bound(G.T, X.double().T, 2050), "dW")


def test_kept_gradients_that_are_not_wanted_and_no_rows():
    a, X, X8, D, D8 = kept(70, 90, 50, "fff", "tanh", 5)
    want = run_kept(a, X8, D8)
    ws = torch.full((M.mgrit_affine_kept_workspace_bytes(a.p),), 0xFF, dtype=torch.uint8, device="cuda")
    for i in range(3):
        out = [torch.full_like(t, float("nan")) if j == i else None for j, t in enumerate(want)]
        M.mgrit_affine_kept_backward(a.p, X8 if i == 1 else None, a.W if i == 0 else None, D8, a.dY, *out, ws)
        near(out[i], want[i].double(), 64 * 2.0 ** -23 * float(want[i].abs().max()), i)     # (it may take another order of sums alone)
    z = M.make_affine(M=0, K=5, F=4)
    dW, db = torch.full((4, 5), 1.0, device="cuda"), torch.full((4,), 1.0, device="cuda")
    M.mgrit_affine_kept_backward(z, None, None, None, None, None, dW, db, None)
    assert not bool(dW.any()) and not bool(db.any())


def test_kept_replays():
    a, X, X8, D, D8 = kept(300, 257, 130, "fbf", "tanh", 6)
    n = M.mgrit_affine_kept_workspace_bytes(a.p)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    px = M.make_packed(rows=300, cols=257, format=M.MGRIT_MX8)
    out = [a.new((a.rows, a.K)), a.new((a.F, a.K)), a.new((a.F,))]

    def go():
        M.mgrit_pack(px, a.X, X8)
        M.mgrit_affine_kept_backward(a.p, X8, a.W, D8, a.dY, *out, ws)

    go()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        go()
    for replay in range(3):
        a.X.copy_(normal(a.X.shape, 1.0, "f", 70 + replay))
        go()
        want = [t.clone() for t in out]
        for t in out:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(out, want)), replay

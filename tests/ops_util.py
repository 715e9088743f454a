"""Plain 64-bit forms of the operators around the solver, and bounds of what float sums may be off, from the operands."""
import torch

import paper_2007_07336_amd as M

TYPES = {"f": torch.float32, "b": torch.bfloat16}
KIND = {"f": M.MGRIT_FP32, "b": M.MGRIT_BF16}
ACT = {"tanh": M.MGRIT_ACT_TANH, "relu": M.MGRIT_ACT_RELU, "identity": M.MGRIT_ACT_IDENTITY}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}        # torch.finfo(t).eps / 2
TINY = 2.0 ** -126                                                   # below it results may be flushed to zero


def normal(shape, std=1.0, t="f", seed=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g, dtype=torch.float64) * std).to(TYPES[t]).cuda()


def sum_bound(A, B, terms):
    """Of sum_k A[i, k] B[j, k] in float, in any order: a step 2^-23 (matrix instructions may cut instead of rounding) for each of
    `terms` additions and a few more for products that are put together from parts, relative to the sum of the magnitudes."""
    return (terms + 8) * 2.0 ** -23 * (A.abs() @ B.abs().T) + terms * TINY


def near(got, want, bound, what):
    """|got - want| <= bound + rounding to got's type, entry by entry; NaN and infinities in the same places."""
    g, w = got.double(), want.double()
    assert got.shape == want.shape, what
    assert torch.equal(torch.isnan(g), torch.isnan(w)), what
    fine = torch.isfinite(w)
    assert torch.equal(g[~fine & ~torch.isnan(w)], w[~fine & ~torch.isnan(w)]), what
    b = bound if torch.is_tensor(bound) else torch.full_like(w, bound)
    over = ((g - w).abs() - (b + HALF[got.dtype] * (w.abs() + b) + TINY))[fine]
    assert over.numel() == 0 or float(over.max()) <= 0.0, (what, float(over.max()), float((g - w).abs()[fine].max()))


class Affine:
    """One layer with random values, its calls, and its results in 64 bits."""

    def __init__(self, rows, K, F, types="fff", act="identity", scale=1.0, bias=True, residual=False, seed=0):
        self.rows, self.K, self.F, self.act, self.scale, self.types = rows, K, F, act, scale, types
        x, w, y = types
        self.p = M.make_affine(M=rows, K=K, F=F, act=ACT[act], xtype=KIND[x], wtype=KIND[w], ytype=KIND[y], scale=scale)
        self.X, self.W = normal((rows, K), 1.0, x, seed + 1), normal((F, K), K ** -0.5, w, seed + 2)
        self.b = normal((F,), 0.3, "f", seed + 3) if bias else None
        self.R = normal((rows, F), 1.0, y, seed + 4) if residual else None
        self.dY = normal((rows, F), 1.0, y, seed + 5)
        n = max(M.mgrit_affine_workspace_bytes(self.p), M.mgrit_affine_backward_workspace_bytes(self.p))
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None      # NaN wherever it is read unwritten

    def new(self, shape, t="f"):
        return torch.full(shape, float("nan"), dtype=TYPES[t], device="cuda")

    def forward(self, factor=False, **kw):
        Y, D = self.new((self.rows, self.F), self.types[2]), self.new((self.rows, self.F), self.types[2]) if factor else None
        M.mgrit_affine_forward(self.p, self.X, self.W, self.b, self.R, Y, D, self.ws, **kw)
        return Y, D

    def backward(self, D, **kw):
        dX, dW, db = self.new((self.rows, self.K), self.types[0]), self.new((self.F, self.K)), self.new((self.F,))
        M.mgrit_affine_backward(self.p, self.X, self.W, D, self.dY, dX, dW, db, self.ws, **kw)
        return dX, dW, db

    def check_forward(self, factor=False):
        Y, D = self.forward(factor)
        X, W = self.X.double(), self.W.double()
        z = X @ W.T
        zb = sum_bound(X, W, self.K)
        if self.b is not None:
            z = z + self.b.double()
            zb = zb + 2.0 ** -23 * z.abs()
        s, what = self.scale, (self.rows, self.K, self.F, self.types, self.act)
        if self.act == "tanh":                       # slope at most 1; its own at most 0.77; 4 steps for the function itself
            y, d = torch.tanh(z), 1.0 / torch.cosh(z) ** 2
            yb, db = zb + 2.0 ** -21 * y.abs(), zb + 2.0 ** -20 * d
        elif self.act == "relu":
            y, d, yb, db = torch.relu(z), (z > 0).double(), zb, (z.abs() <= zb).double()     # undecided at zero
        else:
            y, d, yb, db = z, torch.ones_like(z), zb, torch.zeros_like(z)
        r = self.R.double() if self.R is not None else torch.zeros_like(z)
        near(Y, r + s * y, abs(s) * (yb + 2.0 ** -23 * y.abs()), ("Y",) + what)
        if factor:
            near(D, s * d, abs(s) * (db + 2.0 ** -23 * d), ("D",) + what)
        return Y, D

    def check_backward(self, D):
        dX, dW, db = self.backward(D)
        G = self.dY.double() * (D.double() if D is not None else self.scale)
        what = (self.rows, self.K, self.F, self.types, self.act, D is not None)
        X, W = self.X.double(), self.W.double()
        # G itself: a product of floats rounds once; of the scale once more
        near(dX, G @ W, sum_bound(G, W.T, self.F + 2), ("dX",) + what)
        near(dW, G.T @ X, sum_bound(G.T, X.T, self.rows + 2), ("dW",) + what)
        near(db, G.sum(0), (self.rows + 4) * 2.0 ** -23 * G.abs().sum(0) + self.rows * TINY, ("db",) + what)
        return dX, dW, db

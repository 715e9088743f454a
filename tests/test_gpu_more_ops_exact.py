"""Packed layers, kept activations and block norms where a bound by the number of terms says little: whole numbers whose sums are exact, and long rows by
the sums that are formed."""
import pytest
import torch

import paper_2007_07336_amd as M
from tests.ops_util import ACT, HALF, KIND, TINY, TYPES, near
from tests.test_gpu_block_norm import Block
from tests.test_gpu_norm_rows import serial
from tests.test_gpu_packed import packed, unpacked

pytestmark = pytest.mark.gpu
NAN = float("nan")


def whole(shape, values, seed, t="f"):
    """Entries drawn from `values`."""
    g = torch.Generator().manual_seed(seed)
    return torch.tensor(values, dtype=torch.float64)[torch.randint(0, len(values), shape, generator=g)].to(TYPES[t]).cuda()


def places(n, K, seed):
    """About n columns: both ends, the ends of slabs of 256 and of blocks of 32 in the middle, and any."""
    g = torch.Generator().manual_seed(seed)
    some = [0, 1, 31, 32, 255, 256, K // 2 // 256 * 256 - 1, K // 2 // 256 * 256, K // 256 * 256 - 1, K // 256 * 256, K - 33, K - 2, K - 1]
    return torch.unique(torch.tensor([k for k in some if 0 <= k < K] + torch.randint(0, K, (n,), generator=g).tolist())).cuda()


def not_anything(got, want, bound, what):
    """near, and nine entries of ten would be told from nothing (so from the other sign)."""
    near(got, want, bound, what)
    told = want.abs() > bound + HALF[got.dtype] * (want.abs() + bound) + TINY
    assert float(told.double().mean()) > 0.9, what


# -------------------------------------------------------------------------------------------- sums without rounding
LARGE = [(1, 1 << 22, 3), (3, (1 << 22) - 5, 70), (70, 1 << 20, 5), (2, 40, 200_000), (300, 20, 100_000), (20_000, 33, 40), (100_000, 300, 3), (65, 30_000, 200), (17, 70_000, 90)]


@pytest.mark.parametrize("rows,K,F", LARGE)
@pytest.mark.parametrize("form", ["bf16", "mx4"])
@pytest.mark.parametrize("x", ["f", "b"])
def test_packed_layers_of_whole_numbers(rows, K, F, form, x):
    """At most 300 of a row's entries are not zero: sums of at most 300 * 4 * 6 whole numbers, and of the bias, are floats in any order."""
    X = torch.zeros((rows, K), dtype=TYPES[x], device="cuda")
    at = places(270, K, rows)
    X[:, at] = whole((rows, len(at)), [-4, -3, -2, -1, 0, 1, 2, 3, 4], 1, x)
    w, W = packed(whole((F, K), [-6, -4, -3, -2, -1, 0, 1, 2, 3, 4, 6], 2, "b"), "mx4")
    b = whole((F,), [-5, 0, 7], 3)
    p = M.make_affine_packed(M=rows, K=K, F=F, act=M.MGRIT_ACT_IDENTITY, xtype=KIND[x], xformat=M.MGRIT_MX4 if form == "mx4" else M.MGRIT_BF16)
    n = M.mgrit_affine_packed_workspace_bytes(p)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    Y = torch.full((rows, F), NAN, device="cuda")
    M.mgrit_affine_packed_forward(p, X, W, b, None, Y, None, ws)
    Xv, Wv = X[:, at].double(), torch.empty((F, len(at)), dtype=torch.float64, device="cuda")
    Wv.copy_(unpacked(w, W, "b")[:, at])
    if form == "mx4":                                              # (numbers up to 4 keep their value in a block whose largest is one of them)
        assert torch.equal(unpacked(*packed(X, "mx4"), x)[:, at], X[:, at])
    want = Xv @ Wv.T + b.double()
    assert torch.equal(Y.double(), want) and float((want != 0).double().mean()) > 0.5


@pytest.mark.parametrize("rows,K,F", [(20, 24, (1 << 20) + 3), (3, 300, 10), (300, 257, 16), (520, 1031, 70), (40, 30_000, 300)])
@pytest.mark.parametrize("act", ["tanh", "identity"])
@pytest.mark.parametrize("types", ["fff", "bbb", "fbf"])
def test_kept_activations_of_whole_numbers(rows, K, F, act, types):
    """dY has at most 300 entries that are not zero in a row, sums of 600 * 4 * 4 * 3 are exact; the first size is too wide for the tiles that read 8 bits."""
    p = M.make_affine(M=rows, K=K, F=F, act=ACT[act], xtype=KIND[types[0]], wtype=KIND[types[1]], ytype=KIND[types[2]], scale=0.5)
    X, W = whole((rows, K), [-3, -2, -1, 0, 1, 2, 3], 1, types[0]), whole((F, K), [-4, -2, -1, 0, 1, 3], 2, types[1])
    dY, at = torch.zeros((rows, F), dtype=TYPES[types[2]], device="cuda"), places(270, F, 3)
    dY[:, at] = whole((rows, len(at)), [-4, -3, -1, 0, 1, 2, 4], 4, types[2])
    D = whole((rows, F), [0, 1, 2, 3], 5, types[2]) if act == "tanh" else None
    X8, D8 = packed(X, "mx8")[1], packed(D, "mx8")[1] if D is not None else None
    n = M.mgrit_affine_kept_workspace_bytes(p)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None
    dX, dW, db = (torch.full(s, NAN, dtype=TYPES[t], device="cuda") for s, t in (((rows, K), types[0]), ((F, K), "f"), ((F,), "f")))
    M.mgrit_affine_kept_backward(p, X8, W, D8, dY, dX, dW, db, ws)
    G = dY.double() * (D.double() if D is not None else 0.5)
    want = G @ W.double()
    assert torch.equal(dX, want.to(dX.dtype)) and float((want != 0).double().mean()) > 0.5
    assert torch.equal(dW[at].double(), G[:, at].T @ X.double()) and torch.equal(db.double(), G.sum(0))
    rest = torch.ones(F, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert not bool(dW[rest].any())


# -------------------------------------------------------------------------------------------- norms of long rows
class Summed(Block):
    """Its bounds take the additions that are made one behind the other in place of all of a row's."""

    def steps(self):
        return (serial(self.q) + 24) * 2.0 ** -23

    def exact_backward(self, S, dS):
        """Columns: a workgroup's rows, of 256 workgroups or more if there are as many rows, six steps where several rows share a wavefront, then
        the workgroups (2048 at most) by 32 and their 32 sums."""
        want, bound = super().exact_backward(S, dS)
        e, chain = 2.0 * self.steps(), -(-self.rows // 256) + 6 + 64 + 32
        less = (e + chain * 2.0 ** -23) / (e + (self.rows + 8) * 2.0 ** -23)
        return want, {k: v * min(less, 1.0) + TINY if v.dim() == 1 else v for k, v in bound.items()}

    def check_all(self):
        S, _ = self.check_forward()
        got = self.backward(S)
        want, bound = self.exact_backward(S, self.dS)
        for k, w in want.items():
            not_anything(got[k], w, bound[k], (k, self.rows, self.q, self.kind, self.types))


@pytest.mark.parametrize("rows,q", [(3, 100_003), (2, 1_000_000), (5, 20_011), (700, 9001), (40, 6001), (3000, 130)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("types", ["ff", "fb", "bb"])
def test_norms_of_long_rows(rows, q, kind, types):
    Summed(rows, q, kind, "feature", types, seed=q).check_all()

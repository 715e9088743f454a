"""Packed weights and kept activations with blocks that are NaN: they stay in their columns and rows."""
import math

import pytest
import torch

import paper_2007_07336_amd as M
from tests.ops_util import KIND, TYPES
from tests.test_gpu_more_ops_exact import whole
from tests.test_gpu_packed import PackedLayer, packed, unpacked

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.mark.parametrize("form", ["bf16", "mx4"])
@pytest.mark.parametrize("rows", [1, 3, 17, 40, 64, 70, 600])
@pytest.mark.parametrize("act", ["tanh", "relu"])
def test_weights_that_are_not_finite_stay_in_their_columns(form, rows, act):
    """In the first block, in the middle and in the last, ragged one, of a contraction that several workgroups share (few rows)."""
    a = PackedLayer(rows, 2083, 83, "f", form, "f", act, seed=rows)
    W = unpacked(M.make_packed(rows=83, cols=2083, format=M.MGRIT_MX4), a.W, "f")
    _, a.W = packed(W, "mx4")
    want, _ = a.run()
    bad = [5, 16, 40, 82]
    W[5, 0], W[16, 1000], W[40, 2082], W[82, 2079] = NAN, math.inf, -math.inf, NAN
    _, a.W = packed(W, "mx4")
    got, _ = a.run()
    fine = torch.ones(83, dtype=torch.bool)
    fine[bad] = False
    assert bool(torch.isnan(got[:, bad]).all()) and torch.equal(got[:, fine], want[:, fine])


@pytest.mark.parametrize("rows,K,F", [(3, 300, 10), (300, 257, 16), (33, 2000, 9), (130, 520, 260), (520, 1031, 70), (20, 24, (1 << 20) + 3)])
@pytest.mark.parametrize("types", ["fff", "bbb", "fbf"])
def test_kept_blocks_that_are_not_finite_stay_in_theirs(rows, K, F, types):
    p = M.make_affine(M=rows, K=K, F=F, act=M.MGRIT_ACT_TANH, xtype=KIND[types[0]], wtype=KIND[types[1]], ytype=KIND[types[2]], scale=0.5)
    X, W = whole((rows, K), [-1.5, -1, 0.5, 1, 2], 1, types[0]), whole((F, K), [-1, 0.5, 1], 2, types[1])
    dY, D = whole((rows, F), [-1, 0.25, 1], 3, types[2]), whole((rows, F), [0.25, 0.5], 4, types[2])
    n = M.mgrit_affine_kept_workspace_bytes(p)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None

    def run():
        out = [torch.full(s, NAN, dtype=TYPES[t], device="cuda") for s, t in (((rows, K), types[0]), ((F, K), "f"), ((F,), "f"))]
        M.mgrit_affine_kept_backward(p, packed(X, "mx8")[1], W, packed(D, "mx8")[1], dY, *out, ws)
        return out

    clean = run()
    block = lambda at, n: torch.arange(n, device="cuda") // 32 == at // 32                         # noqa: E731
    X[rows - 1, K - 1] = NAN                                       # (in the last, ragged block)
    got = run()
    cols = block(K - 1, K)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[2], clean[2])
    assert bool(torch.isnan(got[1][:, cols]).all()) and torch.equal(got[1][:, ~cols], clean[1][:, ~cols])
    X[rows - 1, K - 1] = 1.0
    clean = run()
    D[1, F - 1] = math.inf
    got, outs = run(), block(F - 1, F)
    others = torch.arange(rows, device="cuda") != 1
    assert bool(torch.isnan(got[0][1]).all()) and torch.equal(got[0][others], clean[0][others])
    assert bool(torch.isnan(got[1][outs]).all()) and torch.equal(got[1][~outs], clean[1][~outs])
    assert bool(torch.isnan(got[2][outs]).all()) and torch.equal(got[2][~outs], clean[2][~outs])

"""Block norms of rows that are hard for floats: without deviation, with a small one beside a large mean, and of entries whose squares no float holds."""
import math

import pytest
import torch

import paper_2007_07336_amd as M
from tests.ops_util import near, normal
from tests.test_gpu_block_norm import Block, norm_of

pytestmark = pytest.mark.gpu
# one size for every form: lanes of a wavefront, a wavefront, workgroups with one and two vectors a thread, rows that are read again
SIZES = [3, 7, 57, 100, 250, 500, 1000, 2003, 4001, 8001, 12007, 20011]


def serial(q):
    """Additions one behind the other in a sum over a row: a thread's entries, six steps in a wavefront, one wavefront after another."""
    return 8 * -(-q // 8192 if q > 8192 else 1) * (2 if 4096 < q <= 16384 else 1) + 6 + 16


@pytest.mark.parametrize("q", SIZES)
@pytest.mark.parametrize("types", ["ff", "bb"])
def test_rows_without_deviation(q, types):
    """Their mean is each of their entries, so there is nothing left of them: exactly zero beside eps, NaN without it."""
    # (in floats, values that no power of two divides evenly by, and one whose sum no float holds)
    values = torch.tensor([0.1, -1.0 / 3.0, 10000.1, 7.7e8, 3.0e38, 0.0, 1.0e-3])
    b = Block(len(values), q, "layer", "feature", types, eps=1.0e-6, seed=q)
    b.f.copy_(values[:, None].expand_as(b.f))
    b.r.copy_(values.flip(0)[:, None].expand_as(b.r))
    S, Y = b.forward()
    assert torch.equal(S, b.r) and not bool(Y.any())
    got = b.backward(S)
    assert not any(bool(got[k].any()) for k in ("dgate", "dpost", "dpre"))
    assert bool(torch.isfinite(got["df"]).all()) and bool(torch.isfinite(got["dr"]).all())
    # d (h - mean h) with d = 1 / sqrt(eps): 2^-24 of the magnitudes for each addition of a sum's longest chain, 8 for the operations around it
    h = b.dY.double() * b.pre.double()
    d = 1.0 / math.sqrt(torch.tensor(1.0e-6).item())
    e = (serial(q) + 8) * 2.0 ** -24
    near(got["dr"], b.dS.double() + d * (h - h.mean(1, keepdim=True)), e * (b.dS.double().abs() + d * (h.abs() + h.abs().mean(1, keepdim=True))), ("dr", q))
    z = Block(3, q, "layer", "none", types, post=False, eps=0.0, seed=q)
    z.f.copy_(values[:3, None].expand_as(z.f))
    z.r.copy_(values[:3, None].expand_as(z.r))
    S, Y = z.forward()
    assert bool(torch.isfinite(S).all()) and bool(torch.isnan(Y).all())


@pytest.mark.parametrize("q", SIZES[1:])
@pytest.mark.parametrize("center", [1000.0, 0.07])
def test_small_deviations_beside_a_large_mean(q, center):
    """Entries 1000 +- 0.01: their deviations have 7 bits left of the entries' 24, and keep them; 0.07 +- 0.01, a mean just small enough to be taken as it is."""
    b = Block(5, q, "layer", "none", "ff", pre=False, eps=1.0e-6, scale=1.0, seed=q)
    b.f.copy_(center + normal((5, q), 0.01, "f", q))
    b.r.zero_()
    b.post.fill_(1.0)
    S, _ = b.forward()
    want, dev = norm_of(b.f.double(), "layer", b.eps)
    # A mean is off by a step of 2^-24 for each addition of the longest chain and three for the quotient and its own rounding, of the mean magnitude of what it is
    # the mean of: the entries, at most 9 deviations, or (of a larger one) the deviations from the first mean, which are exact.  Those are larger than the
    # true ones by what the first mean is off, (44 + 3) 2^-24 1000 at most: a quarter of a deviation, less than the largest of the true ones.
    mean = lambda t: t.mean(1, keepdim=True)                                                       # noqa: E731
    size = mean(b.f.double().abs()) * dev
    off = (serial(q) + 4) * 2.0 ** -24 * (mean(want.abs()) + want.abs().max(1, keepdim=True).values + torch.where(size < 9, size, 0.0))
    # half of the relative error of a sum of positive terms goes to the whole row
    near(S, want, (serial(q) + 8) * 2.0 ** -24 * want.abs() + off * (1.0 + want.abs()), ("S", q))
    got = b.backward(S)
    dn = b.dS.double()
    df = dev * (dn - want * mean(dn * want) - mean(dn))
    mag = dev * (dn.abs() + want.abs() * mean((dn * want).abs()) + mean(dn.abs()))
    moved = dev * off * (mean((dn * want).abs()) * (1.0 + want.abs()) + want.abs() * mean(dn.abs()) * (1.0 + want.abs()))
    near(got["df"], df, 2 * (serial(q) + 12) * 2.0 ** -24 * mag + moved + dev * off * dn.abs(), ("df", q))


@pytest.mark.parametrize("q", SIZES[1:])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("size", [1.0e-26, 1.0e-22, 1.0e20, 1.0e36])
def test_rows_whose_squares_no_float_holds(q, kind, size):
    """Without eps a row's norm does not depend on its size: the rows beside one that is `size` times as large."""
    s = 2.0 ** round(math.log2(size))
    b = Block(4, q, kind, "feature", "ff", eps=0.0, scale=1.0, seed=q)
    a = Block(4, q, kind, "feature", "ff", eps=0.0, scale=1.0, seed=q)
    a.f[1] *= s
    a.f[3] *= s
    for x in (a, b):
        x.r.zero_()
    (S, Y), (S1, Y1) = b.forward(), a.forward()
    assert torch.equal(S, S1) and torch.equal(Y, Y1)               # (a power of two changes no rounding)
    a.dS, a.dY = b.dS, b.dY
    want, got = b.backward(S), a.backward(S1)
    for k in ("dr", "dgate", "dpost", "dpre"):
        assert torch.equal(want[k], got[k]), k
    assert torch.equal(got["df"][[0, 2]], want["df"][[0, 2]])
    if s > 1:                                                      # (their gradients are as much smaller, some below the least float)
        near(got["df"][[1, 3]], want["df"][[1, 3]].double() / s, 2.0 ** -126, ("df", q))
    # the stream's own size
    a, b = (Block(4, q, kind, "none", "ff", post=False, eps=0.0, scale=1.0, seed=q) for _ in range(2))
    a.f *= s
    a.r *= s
    (S, Y), (S1, Y1) = b.forward(), a.forward()
    assert torch.equal(S * s, S1) and torch.equal(Y, Y1)
    b.dS.zero_()
    a.dS.zero_()
    want, got = b.backward(S), a.backward(S1)
    assert torch.equal(want["dpre"], got["dpre"])
    if s > 1:
        near(got["dr"], want["dr"].double() / s, 2.0 ** -126, ("dr", q))


@pytest.mark.parametrize("q", SIZES[1:])
@pytest.mark.parametrize("size", [-90, -105, -113])
def test_rows_of_the_smallest_floats(q, size):
    """Entries of 2^-113: those near zero have few bits, and their mean keeps what there is."""
    b = Block(4, q, "layer", "none", "ff", pre=False, eps=0.0, scale=1.0, seed=q)
    b.f.copy_(0.5 + b.f).mul_(2.0 ** size)
    b.r.zero_()
    b.post.fill_(1.0)
    S, _ = b.forward()
    x = b.f.double() * 2.0 ** -size                                # (in 64 bits and so in their own)
    want, dev = norm_of(x, "layer", 0.0)
    # a step for each addition of the longest chain and four more, of the deviations' magnitudes (see above); half of 2^-149 for each addition of all, the mean and a
    # difference to it
    mean = lambda t: t.mean(1, keepdim=True)                                                       # noqa: E731
    off = (serial(q) + 4) * 2.0 ** -24 * (mean(want.abs()) + want.abs().max(1, keepdim=True).values + mean(x.abs()) * dev) + (q + 100) * 2.0 ** (-150 - size) * dev
    near(S, want, (serial(q) + 8) * 2.0 ** -24 * want.abs() + off * (1.0 + want.abs()), ("S", q))
    got = b.backward(S)
    # df is beyond the largest float here; dpost is a sum of dS x^
    near(got["dpost"], (b.dS.double() * want).sum(0), (b.dS.double().abs() * (off * (1.0 + want.abs()) + (serial(q) + 14) * 2.0 ** -24 * want.abs())).sum(0), ("dpost", q))

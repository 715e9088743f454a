"""End layers (mgrit_affine_forward, mgrit_affine_backward) against 64-bit products, entry by entry, with bounds that follow
from the operands and the number of additions."""
import pytest
import torch

import paper_2007_07336_amd as M
from tests.ops_util import TINY, Affine, normal, near, sum_bound

pytestmark = pytest.mark.gpu

# rows, inputs, outputs: single values, rows and columns; sizes around 16, 32, 64 and 128; odd ones; heads with few classes; long sums
SHAPES = [(1, 1, 1), (1, 7, 3), (3, 1, 5), (2, 9, 1), (5, 33, 10), (16, 64, 16), (17, 65, 15), (31, 31, 33), (32, 128, 64), (33, 100, 65),
          (64, 256, 10), (65, 257, 129), (100, 784, 96), (128, 64, 127), (1, 1000, 500), (4, 2049, 10), (129, 30, 300), (257, 515, 70),
          (7, 5000, 2), (300, 3, 3)]
TYPES = ["fff", "bbb", "fbf", "bbf", "ffb", "bff"]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,K,F", SHAPES)
def test_forward(rows, K, F, types):
    Affine(rows, K, F, types, "identity").check_forward()
    Affine(rows, K, F, types, "tanh", 0.25, residual=True, seed=10).check_forward(factor=True)
    Affine(rows, K, F, types, "relu", -1.5, bias=False, seed=20).check_forward(factor=True)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,K,F", SHAPES)
def test_backward(rows, K, F, types):
    Affine(rows, K, F, types, "identity", 0.75).check_backward(None)
    a = Affine(rows, K, F, types, "tanh", 0.5, seed=10)
    a.check_backward(a.forward(factor=True)[1])


# sizes that the kernels for many rows, wide layers and long sums take
@pytest.mark.parametrize("types", ["fff", "bbb", "fbf", "bbf"])
@pytest.mark.parametrize("rows,K,F", [(512, 512, 512), (513, 520, 500), (1024, 256, 384), (300, 1111, 777), (2048, 64, 256), (256, 2048, 1000),
                                      (1000, 704, 1290), (32, 4096, 4096), (32, 20000, 10), (2000, 1024, 10), (640, 10, 2000), (16, 520, 9000)])
def test_large(rows, K, F, types):
    a = Affine(rows, K, F, types, "tanh", 0.5, residual=True)
    _, D = a.check_forward(factor=True)
    a.check_backward(D)
    Affine(rows, K, F, types, "identity", seed=3).check_backward(None)


def test_gradients_against_differences():
    """d/dt of the sum of dY * Y along random directions of X, W and b, from float64 differences of the plain form."""
    a = Affine(37, 50, 21, "fff", "tanh", 0.5)
    dX, dW, db = a.backward(a.forward(factor=True)[1])

    def value(t, vX, vW, vb):
        z = (a.X.double() + t * vX) @ (a.W.double() + t * vW).T + a.b.double() + t * vb
        return float((a.dY.double() * 0.5 * torch.tanh(z)).sum())

    for seed in range(4):
        vX, vW, vb = (normal(t.shape, 1.0, "f", 100 + 3 * seed + i).double() for i, t in enumerate((a.X, a.W, a.b)))
        h = 1e-5
        want = (value(h, vX, vW, vb) - value(-h, vX, vW, vb)) / (2 * h)
        got = float((dX.double() * vX).sum() + (dW.double() * vW).sum() + (db.double() * vb).sum())
        size = float((dX.double() * vX).abs().sum() + (dW.double() * vW).abs().sum() + (db.double() * vb).abs().sum())
        # sums of at most 50 + 2 products; the differences are off by h^2 of a third derivative below the size, and 1e-16 / h
        assert abs(got - want) <= (60 * 2.0 ** -23 + 1e-8) * size


def test_outputs_that_are_not_wanted():
    a = Affine(40, 72, 33, "fff", "identity")
    dX, dW, db = a.backward(None)
    for keep in ("dX", "dW", "db"):
        o = {"dX": a.new((40, 72)), "dW": a.new((33, 72)), "db": a.new((33,))}
        M.mgrit_affine_backward(a.p, a.X if keep == "dW" else None, a.W if keep == "dX" else None, None, a.dY,
                                *(o[k] if k == keep else None for k in ("dX", "dW", "db")), a.ws)
        assert torch.equal(o[keep], {"dX": dX, "dW": dW, "db": db}[keep])


@pytest.mark.parametrize("types,rows,K,F", [("fff", 70, 130, 90), ("bbb", 600, 512, 512), ("fbf", 8, 4096, 10)])
def test_residual_may_be_the_output(types, rows, K, F):
    a = Affine(rows, K, F, types, "tanh", residual=True)
    Y, _ = a.forward()
    R = a.R.clone()
    M.mgrit_affine_forward(a.p, a.X, a.W, a.b, R, R, None, a.ws)
    assert torch.equal(R, Y)


@pytest.mark.parametrize("types", ["fff", "bbb", "fbf"])
@pytest.mark.parametrize("rows,K,F", [(6, 40, 10), (130, 200, 150), (512, 512, 512), (32, 4096, 64)])
def test_infinities_and_nan_stay_in_their_rows_and_columns(rows, K, F, types):
    a = Affine(rows, K, F, types)
    a.X[1, 3] = float("inf")
    a.X[2, 0] = float("nan")
    a.W[5, 7] = float("-inf")
    a.dY[4, 2] = float("inf")
    Y, _ = a.forward()
    z = a.X.double() @ a.W.double().T + a.b.double()
    fine = torch.isfinite(z)
    bound = sum_bound(a.X.double().nan_to_num(0, 0, 0), a.W.double().nan_to_num(0, 0, 0), K) + 2.0 ** -22 * z.abs().nan_to_num(0, 0, 0)
    near(Y, z, torch.where(fine, bound, 0.0), "Y")
    dX, dW, db = a.backward(None)
    for got, want in ((dX, a.dY.double() @ a.W.double()), (dW, a.dY.double().T @ a.X.double()), (db, a.dY.double().sum(0))):
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
        assert torch.equal(got[torch.isinf(want)].double(), want[torch.isinf(want)])


@pytest.mark.parametrize("size", [1e-30, 1e-18, 1e18, 3e37])
@pytest.mark.parametrize("rows,K,F", [(40, 60, 30), (512, 512, 512)])
def test_large_and_small_magnitudes(rows, K, F, size):
    """Operands far from one: float sums keep their relative accuracy as long as products and sums are normal numbers."""
    a = Affine(rows, K, F, "fff", "identity", bias=False)
    a.X.mul_(size)
    a.dY.mul_(size / 1e3)
    a.check_forward()
    dX, dW, db = a.new((rows, K)), None, a.new((F,))
    M.mgrit_affine_backward(a.p, None, a.W, None, a.dY, dX, dW, db, a.ws)
    near(dX, a.dY.double() @ a.W.double(), sum_bound(a.dY.double(), a.W.double().T, F + 2), "dX")


def test_no_rows():
    p = M.make_affine(M=0, K=5, F=3)
    e = torch.empty((0, 5), device="cuda")
    y = torch.empty((0, 3), device="cuda")
    dW, db = torch.full((3, 5), 7.0, device="cuda"), torch.full((3,), 7.0, device="cuda")
    W = torch.ones((3, 5), device="cuda")
    assert M.mgrit_affine_forward(p, e, W, None, None, y, None, None) == 0
    assert M.mgrit_affine_backward(p, e, W, None, y, e, dW, db, None) == 0
    assert not dW.any() and not db.any()


@pytest.mark.parametrize("rows,K,F,types", [(7, 33, 10, "fff"), (513, 520, 500, "bbb"), (32, 20000, 10, "fbf"), (300, 1111, 777, "fff"), (1, 512, 3000, "bbb")])
def test_nothing_is_written_past_the_outputs(rows, K, F, types):
    a = Affine(rows, K, F, types, "tanh")

    def guarded(shape, t):
        n, pad = shape[0] * (shape[1] if len(shape) > 1 else 1), 4096
        whole = torch.full((n + 2 * pad,), 7.0, dtype=t, device="cuda")
        return whole, whole[pad:pad + n].view(shape), pad

    o = [guarded((rows, F), a.dY.dtype), guarded((rows, F), a.dY.dtype), guarded((rows, K), a.X.dtype), guarded((F, K), torch.float32),
         guarded((F,), torch.float32)]
    M.mgrit_affine_forward(a.p, a.X, a.W, a.b, None, o[0][1], o[1][1], a.ws)
    M.mgrit_affine_backward(a.p, a.X, a.W, o[1][1], a.dY, o[2][1], o[3][1], o[4][1], a.ws)
    for whole, inner, pad in o:
        assert bool((whole[:pad] == 7.0).all()) and bool((whole[pad + inner.numel():] == 7.0).all())
        assert not bool((inner == 7.0).all())


@pytest.mark.parametrize("rows,K,F,types", [(48, 100, 60, "fff"), (512, 512, 512, "bbb"), (32, 8192, 10, "fbf"), (1, 1024, 4096, "bbb"), (300, 700, 500, "fff")])
def test_captured_calls_replay_with_new_inputs(rows, K, F, types):
    a = Affine(rows, K, F, types, "tanh", 0.5, residual=True)
    Y, D = a.forward(factor=True)
    outs = (Y, D) + a.backward(D)

    def calls():
        M.mgrit_affine_forward(a.p, a.X, a.W, a.b, a.R, Y, D, a.ws)
        M.mgrit_affine_backward(a.p, a.X, a.W, D, a.dY, *outs[2:], a.ws)

    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        calls()
    torch.cuda.synchronize()
    for replay in range(3):
        a.X.copy_(normal((rows, K), 1.0, types[0], 50 + replay))
        a.dY.copy_(normal((rows, F), 1.0, types[2], 60 + replay))
        calls()
        want = [t.clone() for t in outs]
        for t in outs:
            t.fill_(float("nan"))
        a.ws is None or a.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip(outs, want):
            assert torch.equal(t, w), replay


def test_another_stream_and_its_order():
    """Work goes to the stream that is handed over, behind what it holds already."""
    a = Affine(200, 300, 100, "fff", "identity")
    X = a.X.clone()
    want, _ = a.forward()
    a.X.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    Y = a.new((200, 100))
    with torch.cuda.stream(side):
        busy = torch.randn(2048, 2048, device="cuda")
        for _ in range(8):
            busy = busy @ busy * 1e-3
        a.X.copy_(X)
    M.mgrit_affine_forward(a.p, a.X, a.W, a.b, None, Y, None, a.ws, stream=side)
    side.synchronize()
    assert torch.equal(Y, want)


def test_the_same_call_gives_the_same_bits():
    for rows, K, F, types in ((100, 1031, 517, "fff"), (32, 20000, 10, "fbf"), (512, 640, 512, "bbb")):
        a = Affine(rows, K, F, types, "tanh")
        _, D = a.forward(factor=True)
        first = a.backward(D)
        for _ in range(3):
            assert all(torch.equal(x, y) for x, y in zip(first, a.backward(D)))


# float rows against bf16 weights, large enough for products in parts: forward, both gradients, with factors and without
@pytest.mark.parametrize("types", ["fbf", "bbf"])
@pytest.mark.parametrize("rows,K,F", [(1100, 1024, 1000), (300, 1999, 2111), (4096, 520, 600)])
def test_products_in_parts(rows, K, F, types):
    a = Affine(rows, K, F, types, "tanh", 0.5, residual=True)
    _, D = a.check_forward(factor=True)
    a.check_backward(D)
    Affine(rows, K, F, types, "identity", -0.7, seed=3).check_backward(None)


@pytest.mark.parametrize("types,rows,K,F", [("fbf", 1100, 1024, 1000), ("bbb", 600, 512, 520)])
def test_infinities_in_products_in_parts(types, rows, K, F):
    """Not finite where the formula is not, and nowhere else."""
    a = Affine(rows, K, F, types, "tanh")
    D = torch.rand((rows, F), generator=torch.Generator().manual_seed(1)).to(a.dY.dtype).cuda() + 0.1
    a.X[1, 3], a.X[2, 0], a.W[5, 7], a.dY[4, 2], D[9, 9] = (float(v) for v in ("inf", "nan", "-inf", "inf", "nan"))
    big = torch.finfo(torch.float32).max if types[0] == "f" else 3e38
    a.X[7, 7], a.W[5, 8] = big, 0.5                             # next to what bf16 rounds to infinity
    Y = a.new((rows, F), types[2])
    p = M.make_affine(M=rows, K=K, F=F, xtype=a.p.xtype, wtype=a.p.wtype, ytype=a.p.ytype)
    M.mgrit_affine_forward(p, a.X, a.W, None, None, Y, None, a.ws)
    z = a.X.double() @ a.W.double().T
    over = z.abs() > 3.3e38                                      # sums that leave float may do so at any point
    assert torch.equal(torch.isfinite(Y)[~over], torch.isfinite(z)[~over])
    dX, dW, db = a.backward(D)
    G = a.dY.double() * D.double()
    for got, want in ((dX, G @ a.W.double()), (dW, G.T @ a.X.double()), (db, G.sum(0))):
        over = want.abs() > 3.3e38
        assert torch.equal(torch.isfinite(got)[~over], torch.isfinite(want)[~over])


def test_rows_beyond_32_bit_offsets():
    """Contractions and rows whose offsets within a tile pass 2^31 bytes: the plain tile takes them."""
    a = Affine(70, 1100001, 66, "bbb", "tanh", residual=True)
    _, D = a.check_forward(factor=True)
    a = Affine(17, 4300003, 18, "bbb", bias=False)
    a.check_backward(None)


@pytest.mark.parametrize("rows,K,F", [(1, 300000, 1), (70000, 5, 2), (2, 3, 200000), (1, 2, 3), (100000, 20, 20), (19, 1, 70), (70, 70, 1)])
def test_long_and_thin(rows, K, F):
    a = Affine(rows, K, F, "fff", "tanh", 0.5)
    _, D = a.check_forward(factor=True)
    a.check_backward(D)


# two float operands, large enough for products in parts of both; and with a float weight the other types
@pytest.mark.parametrize("types", ["fff", "ffb", "bff"])
@pytest.mark.parametrize("rows,K,F", [(2200, 2100, 2301), (4096, 1024, 2560)])
def test_float_products_in_parts(rows, K, F, types):
    a = Affine(rows, K, F, types, "tanh", 0.5)
    _, D = a.check_forward(factor=True)
    a.check_backward(D)


# few rows on one side against so many on the other that a workgroup takes two blocks of them; aligned rows and odd ones; either side
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("few", [3, 16, 17, 32, 33, 50, 64, 65])
def test_few_rows_against_many(few, types):
    for K in (200, 515):
        Affine(few, K, 8203, types, "tanh", 0.5, residual=True).check_forward(factor=True)
        Affine(8203, K, few, types, "relu", 2.0, bias=False, seed=7).check_forward()
    a = Affine(few, 72, 8203, types, "identity", 0.3, seed=11)
    a.check_backward(None)


@pytest.mark.parametrize("types", ["fff", "bbb", "fbf"])
def test_sizes_around_the_tiles(types):
    """One more and one less than whole tiles and slabs, in every place, so that edges of all three kinds meet."""
    for n in (63, 65, 127, 129, 255, 257):
        for rows, K, F in ((n, 96, 160), (160, n, 130), (130, 160, n), (n, n, n)):
            a = Affine(rows, K, F, types, "tanh", 0.5, seed=n)
            _, D = a.check_forward(factor=True)
            a.check_backward(D)
    Affine(16 * 256 + 1, 64, 16 * 256 - 1, types, "relu", residual=True).check_forward()


@pytest.mark.parametrize("types", ["fff", "bbb", "fbf"])
@pytest.mark.parametrize("M_,K,F,at", [(20, 40, 10, (0, 3)), (70, 300, 10, (64, 9)), (1000, 33, 3, (0, 0)), (5, 40, 50, (2, 0)), (3, 700, 333, (0, 32)),
                                       (1, 9, 17, (0, 0)), (300, 20, 16, (288, 15))])
def test_an_infinite_gradient_in_the_first_row_of_a_chunk(M_, K, F, at, types):
    """Thin gradients: rows behind a chunk's last one take no part, so an infinity stays one where the formula has it."""
    a = Affine(M_, K, F, types)
    a.dY[at] = float("inf")
    dX, dW, db = a.backward(None)
    for got, want in ((dX, a.dY.double() @ a.W.double()), (dW, a.dY.double().T @ a.X.double()), (db, a.dY.double().sum(0))):
        assert torch.isinf(want).any()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
        assert torch.equal(got[torch.isinf(want)].double(), want[torch.isinf(want)])


@pytest.mark.parametrize("many_rows", [True, False])
def test_more_few_rows_workgroups_than_a_launch_has_threads_for(many_rows):
    """2^29 + 5 rows, or columns, of one term each: a product of two bf16 values is exact in float, with the bias it is rounded once."""
    n = (1 << 29) + 5
    v = normal((1 << 14,), 1.0, "b", 1)
    long = torch.empty((n, 1), dtype=torch.bfloat16, device="cuda")
    whole = n // (1 << 14) * (1 << 14)
    long[:whole].view(-1, 1 << 14).copy_(v.expand(whole >> 14, 1 << 14))
    long[whole:, 0] = v[:n - whole]
    one = torch.full((1, 1), 1.625, dtype=torch.bfloat16, device="cuda")
    Y = torch.full((n, 1) if many_rows else (1, n), float("nan"), device="cuda")
    p = M.make_affine(M=n if many_rows else 1, K=1, F=1 if many_rows else n, xtype=1, wtype=1)
    assert M.mgrit_affine_workspace_bytes(p) == 0
    M.mgrit_affine_forward(p, *((long, one) if many_rows else (one, long)), None, None, Y, None, None)
    want = v.float() * 1.625
    flat = Y.view(-1)
    assert bool((flat[:whole].view(-1, 1 << 14) == want).all()) and torch.equal(flat[whole:], want[:n - whole])


def test_more_columns_than_a_launch_has_threads_for():
    """1.5e9 columns of G: its sums over chunks of rows, the chunks' sums and the tiles of dW are each more than 2^32 threads.  Small whole
    numbers, so that every sum is exact; the columns repeat."""
    rows, F, n = 17, 1_500_000_001, 1 << 14
    g = torch.Generator().manual_seed(1)
    v = torch.randint(-8, 9, (rows, n), generator=g).to(torch.bfloat16).cuda()
    X = torch.randint(-8, 9, (rows, 1), generator=g).to(torch.bfloat16).cuda()
    dY = torch.empty((rows, F), dtype=torch.bfloat16, device="cuda")
    whole = F // n * n
    for r in range(rows):
        dY[r, :whole].view(-1, n).copy_(v[r].expand(whole // n, n))
        dY[r, whole:] = v[r, :F - whole]
    p = M.make_affine(M=rows, K=1, F=F, xtype=1, wtype=1, ytype=1)
    ws = torch.empty(M.mgrit_affine_backward_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    dW, db = torch.full((F, 1), float("nan"), device="cuda"), torch.full((F,), float("nan"), device="cuda")
    M.mgrit_affine_backward(p, X, None, None, dY, None, dW, db, ws)
    for got, want in ((db, v.float().sum(0)), (dW[:, 0], (v.float() * X.float()).sum(0))):
        assert bool((got[:whole].view(-1, n) == want).all()) and torch.equal(got[whole:], want[:F - whole])
    del dY, ws, dW, db, got
    torch.cuda.empty_cache()


def _whole(shape, bits, seed):
    """Odd whole numbers of `bits` bits, either sign, as doubles."""
    g = torch.Generator().manual_seed(seed)
    v = torch.randint(1 << (bits - 1), 1 << bits, shape, generator=g, dtype=torch.int64) | 1
    return (v * (2 * torch.randint(0, 2, shape, generator=g) - 1)).double().cuda()


def _picks(rows, cols, value, t, seed):
    """[rows][cols] with one entry of +-value in every row, and the column it is in."""
    g = torch.Generator().manual_seed(seed)
    at = torch.randint(0, cols, (rows,), generator=g).cuda()
    m = torch.zeros((rows, cols), dtype=torch.float64, device="cuda")
    m[torch.arange(rows, device="cuda"), at] = ((2 * torch.randint(0, 2, (rows,), generator=g) - 1).double() * value).cuda()
    return m.to(t)


# Products in parts: every row of one operand picks a single entry of the other, whose 24 bits all have to arrive.  (float rows and bf16
# weights are taken in parts from 1e9 multiplications on, two float operands from 6e9; tiles of 256 and 128, whole and ragged)
PARTED = [("fbf", 1100, 1024, 1000), ("fbf", 4096, 1024, 4096), ("fff", 2200, 2100, 2301), ("fff", 4096, 1024, 2560), ("fbf", 4096, 64, 4096), ("fff", 8200, 96, 8200)]


@pytest.mark.parametrize("exponent,lift", [(0, 0), (-126, 100), (-131, 60), (-149, 80), (-140, 127), (90, -80), (104, 0)])
@pytest.mark.parametrize("types,rows,K,F", PARTED)
def test_every_bit_of_a_float_operand_arrives(types, rows, K, F, exponent, lift):
    """Entries v 2^exponent with v of 24 bits, down to the smallest normal float and up to the largest, times 2^lift."""
    a = Affine(rows, K, F, types, bias=False)
    v = _whole((rows, K), 24, 1) * 2.0 ** exponent
    assert bool((v.float().double() == v).all())
    a.X.copy_(v)
    a.W.copy_(_picks(F, K, 2.0 ** lift, a.W.dtype, 2))
    Y, _ = a.forward()
    assert torch.equal(Y.double(), v @ a.W.double().T)
    if types == "fff":                                             # the other operand, and both gradients
        w = _whole((F, K), 24, 3) * 2.0 ** exponent
        a.W.copy_(w)
        a.X.copy_(_picks(rows, K, 2.0 ** lift, torch.float32, 4))
        assert torch.equal(a.forward()[0].double(), a.X.double() @ w.T)
        g = _whole((rows, F), 24, 5) * 2.0 ** exponent
        a.dY.copy_(g)
        a.W.copy_(_picks(K, F, 2.0 ** lift, torch.float32, 6).T)
        a.X.copy_(_picks(K, rows, 2.0 ** lift, torch.float32, 7).T)
        dX, dW, _ = a.backward(None)
        assert torch.equal(dX.double(), g @ a.W.double()) and torch.equal(dW.double(), g.T @ a.X.double())


@pytest.mark.parametrize("exponent,lift", [(0, 0), (-126, 100), (-140, 100), (100, -60), (111, 0)])
@pytest.mark.parametrize("rows,K,F", [(600, 512, 520), (2048, 1024, 1024)])
def test_every_bit_of_a_product_of_two_bf16_values_arrives(rows, K, F, exponent, lift):
    """G = dY * D has 16 bits and goes into the products as it is."""
    a = Affine(rows, K, F, "bbb", "tanh")
    d = _whole((rows, F), 8, 1) * 2.0 ** -7
    y = _whole((rows, F), 8, 2) * 2.0 ** (exponent + 7)
    a.dY.copy_(y)
    g = y * d
    D = d.bfloat16()
    assert bool((a.dY.double() * D.double() == g).all()) and bool((g.float().double() == g).all())
    a.X.copy_(_picks(K, rows, 2.0 ** lift, torch.bfloat16, 7).T)
    a.W.copy_(_picks(K, F, 2.0 ** lift, torch.bfloat16, 6).T)
    dX, dW, _ = a.backward(D)
    assert torch.equal(dW.double(), g.T @ a.X.double())
    assert torch.equal(dX, (g @ a.W.double()).bfloat16())


@pytest.mark.parametrize("rows,K,F", [(2200, 2100, 2301), (4096, 1024, 2560)])
def test_the_middle_parts_of_both_operands_meet(rows, K, F):
    """12 bits times 12 bits: the parts behind the first of either operand are multiplied with each other, too."""
    a = Affine(rows, K, F, "fff", bias=False)
    v = _whole((rows, K), 12, 1)
    a.X.copy_(v)
    w = _picks(F, K, 1.0, torch.float64, 2) * _whole((F, 1), 12, 3)
    a.W.copy_(w)
    assert torch.equal(a.forward()[0].double(), v @ w.T)


@pytest.mark.parametrize("rows", [1 << 16, 200])
def test_tanh_and_its_slope_near_saturation(rows):
    """Relative errors in steps of 2^-23: the exponential and its correction 1.5, the reciprocal of a rounded sum 1.5, and half a step for
    each product, so 5.5 for 4 e r^2 and at most 4 for (1 - e) r; the result is scaled by 1."""
    z = torch.cat([torch.linspace(-43, 43, rows - 100), torch.linspace(-0.4, 0.4, 90), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 0.35, -0.35, 1e30, -1e30, 88.0, 3e38])])
    X = z[:, None].cuda()
    W, Y, D = torch.ones((1, 1), device="cuda"), torch.empty_like(X), torch.empty_like(X)
    if rows == 200:                                              # columns, with the large tiles' code
        X, W = torch.ones((300, 8), device="cuda"), torch.zeros((rows, 8))
        W[:, 3] = z
        W, Y, D = W.cuda(), torch.empty((300, rows), device="cuda"), torch.empty((300, rows), device="cuda")
    p = M.make_affine(M=X.shape[0], K=X.shape[1], F=W.shape[0], act=M.MGRIT_ACT_TANH)
    ws = torch.empty(M.mgrit_affine_workspace_bytes(p) + 16, dtype=torch.uint8, device="cuda")
    M.mgrit_affine_forward(p, X, W, None, None, Y, D, ws)
    v = (X.double() @ W.double().T)
    e = torch.exp(-2.0 * v.abs())
    near(Y, torch.tanh(v), 4 * 2.0 ** -23 * torch.tanh(v).abs() + TINY, "tanh")
    slope = 4.0 * e / (1.0 + e) ** 2
    near(D, slope, 6 * 2.0 ** -23 * slope + 8 * TINY, "slope")


def test_tanh_of_what_is_not_finite():
    X = torch.tensor([[float("inf")], [float("-inf")], [float("nan")]], device="cuda")
    Y, D = torch.empty_like(X), torch.empty_like(X)
    p = M.make_affine(M=3, K=1, F=1, act=M.MGRIT_ACT_TANH)
    M.mgrit_affine_forward(p, X, torch.ones((1, 1), device="cuda"), None, None, Y, D, None)
    assert Y[:2, 0].tolist() == [1.0, -1.0] and D[:2, 0].tolist() == [0.0, 0.0] and bool(torch.isnan(Y[2]) & torch.isnan(D[2]))


# few rows against many with so long a contraction that every wavefront goes through several slabs: places in LDS are filled again while
# others are read.  Whole 16-byte rows in all types, with whole slabs and without; a contraction shared by workgroups
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("few,many,K", [(3, 8203, 2048), (16, 8203, 2056), (17, 8203, 4096), (32, 8203, 2048), (64, 8203, 2056), (64, 8203, 4104), (16, 500, 9000),
                                        (33, 129, 16384)])
def test_few_rows_with_a_long_contraction(few, many, K, types):
    Affine(few, K, many, types, "tanh", 0.5, residual=True).check_forward(factor=True)
    Affine(many, K, few, types, "relu", 2.0, bias=False, seed=7).check_forward()


@pytest.mark.parametrize("types,rows,K,F", PARTED)
def test_products_near_the_largest_float(types, rows, K, F):
    """Single products in [2^127, 2^128) of values half a bf16 step from the next ones: what the first parts leave is as large as it gets."""
    g = torch.Generator().manual_seed(1)

    def values(shape, odd):                                       # 257 .. 361 (odd) or 129 .. 181, by 2^-8 or 2^-7, either sign
        n = torch.randint(128, 181, shape, generator=g, dtype=torch.int64)
        n = (2 * n + 1).double() / 256 if odd else (n + 1).double() / 128
        return (n * (2 * torch.randint(0, 2, shape, generator=g) - 1).double()).cuda()

    a = Affine(rows, K, F, types, bias=False)
    v = values((rows, K), True) * 2.0 ** 64
    a.X.copy_(v)
    w = _picks(F, K, 1.0, torch.float64, 2) * values((F, 1), types == "fff") * 2.0 ** 63
    a.W.copy_(w)
    want = v @ w.T
    assert bool((a.W.double() == w).all()) and float(want.abs().max()) < 2.0 ** 128 and float(want.abs().min()) >= 2.0 ** 127
    assert torch.equal(a.forward()[0].double(), want)


@pytest.mark.parametrize("types,rows,K,F", PARTED)
def test_products_whose_first_parts_pass_the_largest_float(types, rows, K, F):
    """Values a little below powers of two, which bf16 rounds up to those: the product of the first parts alone is 2^128, the whole one is not."""
    g = torch.Generator().manual_seed(1)

    def values(shape):                                            # 1 - n 2^-12, n = 1 .. 7, either sign
        n = torch.randint(1, 8, shape, generator=g, dtype=torch.int64).double()
        return ((1.0 - n * 2.0 ** -12) * (2 * torch.randint(0, 2, shape, generator=g) - 1).double()).cuda()

    a = Affine(rows, K, F, types, bias=False)
    v = values((rows, K)) * 2.0 ** 65
    a.X.copy_(v)
    w = _picks(F, K, 1.0, torch.float64, 2) * (values((F, 1)) if types == "fff" else 1.0) * 2.0 ** 63
    a.W.copy_(w)
    want = v @ w.T
    assert bool((a.X.bfloat16().double().abs() == 2.0 ** 65).all()) and float(want.abs().max()) < 2.0 ** 128
    assert torch.equal(a.forward()[0].double(), want)


# large products with a short side, where the instructions are chosen by bytes as well: either way, mixed within a backward pass
@pytest.mark.parametrize("types", ["fff", "fbf"])
@pytest.mark.parametrize("rows,K,F", [(6300, 56, 20300), (4100, 300, 5000), (110, 8200, 8300), (8200, 8300, 110), (20000, 200, 600)])
def test_large_products_with_a_short_side(rows, K, F, types):
    a = Affine(rows, K, F, types, "tanh", 0.5, residual=True)
    _, D = a.check_forward(factor=True)
    a.check_backward(D)
    Affine(rows, K, F, types, "identity", 0.7, seed=3).check_backward(None)

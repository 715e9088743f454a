"""Packed arrays, packed layers, block norms and sampling where offsets pass 32 bits, at the longest rows, and two calls at once."""
import pytest
import torch

import paper_2007_07336_amd as M
from tests.ops_util import near, normal, sum_bound
from tests.test_gpu_block_norm import Block
from tests.test_gpu_packed import PackedLayer, kept, packed, run_kept, unpacked, values_of
from tests.test_gpu_sample import call, check, uniform, whole

pytestmark = pytest.mark.gpu


def test_packing_beyond_32_bits():
    rows, cols = 1_100_000, 4096                                   # 4.5e9 values, 9 GB
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    some = [0, 524_287, 524_288, 1_048_575, 1_048_576, rows - 1]
    x[some] = normal((len(some), cols), 1.0, "b", 1)
    for form, name in ((M.MGRIT_MX8, "mx8"), (M.MGRIT_MX4, "mx4")):
        p = M.make_packed(rows=rows, cols=cols, format=form, dtype=M.MGRIT_BF16)
        a = torch.empty(M.mgrit_packed_bytes(p), dtype=torch.uint8, device="cuda")
        M.mgrit_pack(p, x, a)
        y = torch.empty_like(x)
        M.mgrit_unpack(p, a, y)
        assert torch.equal(y[some].cpu().double(), values_of(x[some], name))
        assert int((y != 0).any(1).sum()) == len(some)
        del a, y


def test_sampling_beyond_32_bits():
    B, V = 70_000, 65_536                                          # 4.6e9 logits, 9 GB
    x = torch.zeros((B, V), dtype=torch.bfloat16, device="cuda")
    some = [0, 65_535, 65_536, B - 1]
    x[some] = normal((len(some), V), 2.0, "b", 1)
    u, k, p = torch.full((B,), 0.75, device="cuda"), torch.full((B,), 40, dtype=torch.int32, device="cuda"), torch.full((B,), 0.8, device="cuda")
    index, logprob = call(x, u, None, k, p)
    want, lp = call(x[some].clone(), u[some].clone(), None, k[some].clone(), p[some].clone())
    assert torch.equal(index[some], want) and torch.equal(logprob[some], lp)
    rest = torch.ones(B, dtype=torch.bool, device="cuda")
    rest[some] = False
    assert bool((index[rest] == 24).all())                         # 40 equal ones, 32 of them left, the first beyond three quarters


@pytest.mark.parametrize("dtype,V", [("f", 1_000_003), ("b", 3_000_001)])
def test_sampling_from_very_many_classes(dtype, V):
    x = normal((2, V), 2.0, dtype, 3)
    check(x, uniform(2, 1), k=whole(2, 5, 50, 2))
    check(x, uniform(2, 1), t=uniform(2, 4, 0.5, 1.5), p=uniform(2, 3, 0.3, 0.9))


def test_norms_beyond_32_bits():
    rows, q = 2_200_000, 2048                                      # 4.5e9 entries
    f, r = torch.zeros((rows, q), dtype=torch.bfloat16, device="cuda"), torch.ones((rows, q), dtype=torch.bfloat16, device="cuda")
    some = [0, 1_048_576, 2_097_151, 2_097_152, rows - 1]
    f[some] = normal((len(some), q), 1.0, "b", 1)
    post, pre = 1.0 + normal((q,), 0.1, "f", 2), 1.0 + normal((q,), 0.1, "f", 3)

    def run(m, f, r):
        p = M.make_block_norm(M=m, q=q, stype=M.MGRIT_BF16, ftype=M.MGRIT_BF16, eps=1.0e-5)
        S, Y = torch.empty_like(r), torch.empty_like(f)
        M.mgrit_block_norm_forward(p, f, r, None, post, pre, S, Y)
        df, dr, ws = torch.empty_like(f), torch.empty_like(r), torch.empty(M.mgrit_block_norm_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        M.mgrit_block_norm_backward(p, f, S, None, post, pre, None, Y, df, dr, None, None, None, ws)
        return S, Y, df, dr

    for big, small in zip(run(rows, f, r), run(len(some), f[some].clone(), r[some].clone())):
        assert torch.equal(big[some], small)


@pytest.mark.parametrize("rows,q", [(3, 100_003), (2, 1_000_000)])
def test_norms_of_very_long_rows(rows, q):
    b = Block(rows, q, "layer", "feature", "fb", seed=5)
    S, _ = b.check_forward()
    b.check_backward(S)


@pytest.mark.parametrize("rows,K,F", [(1, 1 << 22, 3), (3, (1 << 22) - 5, 70), (70, 1 << 20, 5), (2, 40, 200_000), (300, 20, 100_000), (20_000, 33, 40), (100_000, 300, 3)])
@pytest.mark.parametrize("form", ["bf16", "mx4"])
def test_packed_layers_of_extreme_shapes(rows, K, F, form):
    PackedLayer(rows, K, F, "b", form, "f", "identity", seed=7).check()


@pytest.mark.parametrize("act", ["tanh", "identity"])
def test_kept_activations_of_a_layer_of_a_million_outputs(act):
    """Too wide for the tiles that read activations in 8 bits: they are unpacked first."""
    rows, K, F = 20, 24, (1 << 20) + 3
    a, X, X8, D, D8 = kept(rows, K, F, "fff", act, 3)
    dX, dW, db = run_kept(a, X8, D8)
    G = a.dY.double() * (D.double() if D is not None else a.scale)
    near(dX, G @ a.W.double(), sum_bound(G, a.W.double().T, F + 2), "dX")
    near(dW, G.T @ X.double(), sum_bound(G.T, X.double().T, rows + 2), "dW")
    near(db, G.sum(0), (rows + 4) * 2.0 ** -23 * G.abs().sum(0) + rows * 2.0 ** -126, "db")


def test_calls_at_once_on_two_streams():
    layers = [PackedLayer(600, 520, 300, "f", "mx4", "f", seed=s) for s in (1, 2)] + [PackedLayer(9, 1000, 300, "f", "bf16", "f", seed=s) for s in (3, 4)]
    blocks = [Block(500, 700, "layer", "feature", "fb", seed=s) for s in (5, 6)]
    Ss = [b.forward()[0] for b in blocks]
    want = [a.run()[0] for a in layers] + [b.backward(S)["dpre"] for b, S in zip(blocks, Ss)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        got = [a.run(stream=streams[i % 2])[0] for i, a in enumerate(layers)] + [b.backward(S, stream=streams[i])["dpre"] for i, (b, S) in enumerate(zip(blocks, Ss))]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)


def test_a_state_inside_a_larger_array_will_do():
    """Rows of a larger array begin at any multiple of 16 bytes; nothing outside them is written."""
    big = normal((9, 4, 20), 1.0, "f", 1)
    f, r = normal((4, 20), 1.0, "f", 2), big[3]
    p = M.make_block_norm(M=4, q=20)
    S, Y = torch.full((6, 4, 20), 7.0, device="cuda"), torch.full((6, 4, 20), 7.0, device="cuda")
    pre = torch.ones(20, device="cuda")
    M.mgrit_block_norm_forward(p, f, r, None, None, pre, S[2], Y[3])
    assert bool((S[[0, 1, 3, 4, 5]] == 7).all()) and bool((Y[[0, 1, 2, 4, 5]] == 7).all())
    near(S[2], r.double() + f.double(), 2.0 ** -23 * (r.double().abs() + f.double().abs()), "S")
    q, a = packed(big[5], "mx8")
    assert torch.equal(unpacked(q, a, "f").cpu().double(), values_of(big[5], "mx8"))
    W, w = packed(normal((6, 20), 0.3, "b", 3), "mx4")
    layer = M.make_affine_packed(M=4, K=20, F=6, xtype=M.MGRIT_FP32, xformat=M.MGRIT_BF16)
    out = torch.full((5, 4, 6), 7.0, device="cuda")
    ws = torch.empty(M.mgrit_affine_packed_workspace_bytes(layer), dtype=torch.uint8, device="cuda")
    M.mgrit_affine_packed_forward(layer, big[7], w, None, None, out[2], None, ws)
    Wv, Xv = unpacked(W, w, "f").double(), big[7].bfloat16().double()
    near(out[2], Xv @ Wv.T, sum_bound(Xv, Wv, 20), "Y")
    assert bool((out[[0, 1, 3, 4]] == 7).all())

"""Packed layers and block norms on another stream in order, on two at once, and gradients in the place of what they are made from."""
import pytest
import torch

import paper_2007_07336_amd as M
from tests.test_gpu_block_norm import Block
from tests.test_gpu_packed import PackedLayer

pytestmark = pytest.mark.gpu
NAN = float("nan")


def test_on_another_stream_in_order():
    """Outputs are filled before the stream's call is allowed to begin, and compared."""
    for form, rows in (("bf16", 5), ("mx4", 5), ("bf16", 200), ("mx4", 700)):
        a = PackedLayer(rows, 520, 300, "f", form, "f", seed=4)
        want, _ = a.run()
        side, out = torch.cuda.Stream(), torch.full_like(want, NAN)
        side.wait_stream(torch.cuda.current_stream())
        M.mgrit_affine_packed_forward(a.p, a.X, a.W, a.b, a.R, out, None, a.ws, stream=side)
        side.synchronize()
        assert torch.equal(out, want), (form, rows)


def test_at_once_on_two_streams_with_outputs_of_their_own():
    layers = [PackedLayer(600, 520, 300, "f", "mx4", "f", seed=s) for s in (1, 2)] + [PackedLayer(9, 1000, 300, "f", "bf16", "f", seed=s) for s in (3, 4)]
    blocks = [Block(500, 700, "layer", "feature", "fb", seed=s) for s in (5, 6)]
    Ss = [b.forward()[0] for b in blocks]
    want = [a.run()[0] for a in layers] + [b.backward(S)["dpre"] for b, S in zip(blocks, Ss)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[torch.full_like(w, NAN) for w in want] for _ in range(4)]            # every round its own
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    for out in got:
        for i, a in enumerate(layers):
            M.mgrit_affine_packed_forward(a.p, a.X, a.W, a.b, a.R, out[i], None, a.ws, stream=streams[i % 2])
        for i, (b, S) in enumerate(zip(blocks, Ss)):
            M.mgrit_block_norm_backward(b.p, b.f, S, b.gate, b.post, b.pre, b.dS, b.dY, None, None, None, None, out[4 + i], b.ws, stream=streams[i])
    torch.cuda.synchronize()
    for r, out in enumerate(got):
        for i, (g, w) in enumerate(zip(out, want)):
            assert torch.equal(g, w), (r, i)


@pytest.mark.parametrize("types", ["fb", "bf", "bb"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("q", [300, 4099, 6000, 8192])
def test_gradients_in_place(q, kind, types):
    """dr in dS' place, df in dY's or f's, for each type."""
    b = Block(7, q, kind, "entry", types, seed=q)
    S, _ = b.forward()
    want = b.backward(S)
    for again in (dict(dS=True, dY=True), dict(f=True)):
        f, dS, dY = b.f.clone(), b.dS.clone(), b.dY.clone()
        df, dr = f if "f" in again else dY, dS if "dS" in again else None
        M.mgrit_block_norm_backward(b.p, f, S, b.gate, b.post, b.pre, dS, dY, df, dr, None, None, None, b.ws)
        assert torch.equal(df, want["df"]) and (dr is None or torch.equal(dr, want["dr"]))

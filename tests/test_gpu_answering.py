"""Packed layers, kept activations, block norms and sampling as they are used together: a training step whose activations are kept in 8 bits
between the passes, and answers from a head with weights in 4 bits."""
import pytest
import torch

import paper_2007_07336_amd as M
from tests.ops_util import near, normal
from tests.test_gpu_block_norm import norm_of
from tests.test_gpu_packed import packed, unpacked
from tests.test_gpu_sample import answer, uniform, whole

pytestmark = pytest.mark.gpu
EPS, STEP = 1.0e-5, 0.5


class Network:
    """A stack of N residual layers, a wide block behind it between norms (S = u^N + STEP gate norm(tanh(u^N Wb^T + bb)) w_post, Y = norm(S) w_pre), a head"""

    def __init__(self, B, q, N, classes):
        f = lambda *s: torch.zeros(s, device="cuda")                                                # noqa: E731
        self.B, self.q, self.N, self.classes = B, q, N, classes
        self.u0, self.labels = normal((B, q), 1.0, "f", 1), torch.randint(0, classes, (B,), generator=torch.Generator().manual_seed(2)).cuda()
        self.par = {"W": normal((N, q, q), q ** -0.5, "f", 3), "b": normal((N, q), 0.3, "f", 4), "Wb": normal((q, q), q ** -0.5, "f", 5),
                    "bb": normal((q,), 0.3, "f", 6), "gate": torch.sigmoid(normal((q,), 1.0, "f", 7)), "post": 1.0 + normal((q,), 0.1, "f", 8),
                    "pre": 1.0 + normal((q,), 0.1, "f", 9), "Wo": normal((classes, q), q ** -0.5, "f", 10), "bo": normal((classes,), 0.3, "f", 11)}
        self.grad = {k: torch.full_like(v, float("nan")) for k, v in self.par.items()}
        self.stack = M.make_problem(N=N, h=1.0 / N, m=4, max_levels=1, relax=0, max_iter=1, layer=0, act=M.MGRIT_ACT_TANH, dtype=0, B=B, q=q)
        self.block = M.make_affine(M=B, K=q, F=q, act=M.MGRIT_ACT_TANH)
        self.norm = M.make_block_norm(M=B, q=q, gate=M.MGRIT_GATE_FEATURE, eps=EPS, scale=STEP)
        self.head = M.make_affine(M=B, K=q, F=classes)
        self.loss = M.make_loss(B=B, V=classes)
        self.keep = M.make_packed(rows=B, cols=q, format=M.MGRIT_MX8)
        room = lambda: torch.zeros(M.mgrit_packed_bytes(self.keep), dtype=torch.uint8, device="cuda")  # noqa: E731
        self.u8, self.D8, self.Y8 = room(), room(), room()
        self.U, self.Lam = f(N + 1, B, q), f(N + 1, B, q)
        self.f, self.D, self.S, self.Y, self.df, self.dr, self.lamN = (f(B, q) for _ in range(7))
        self.logits, self.value = f(B, classes), f(1)
        n = max(M.mgrit_adjoint_workspace_bytes(self.stack), M.mgrit_workspace_bytes(self.stack), M.mgrit_affine_workspace_bytes(self.block),
                M.mgrit_affine_workspace_bytes(self.head), M.mgrit_affine_kept_workspace_bytes(self.block), M.mgrit_affine_kept_workspace_bytes(self.head),
                M.mgrit_block_norm_workspace_bytes(self.norm), M.mgrit_cross_entropy_workspace_bytes(self.loss))
        self.ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def step(self):
        p, g, ws = self.par, self.grad, self.ws
        M.mgrit_fas_forward(self.stack, p["W"], p["b"], self.u0, self.U, ws, want_hist=False)
        u = self.U[self.N]
        M.mgrit_affine_forward(self.block, u, p["Wb"], p["bb"], None, self.f, self.D, ws)
        M.mgrit_pack(self.keep, u, self.u8)
        M.mgrit_pack(self.keep, self.D, self.D8)
        M.mgrit_block_norm_forward(self.norm, self.f, u, p["gate"], p["post"], p["pre"], self.S, self.Y)
        M.mgrit_affine_forward(self.head, self.Y, p["Wo"], p["bo"], None, self.logits, None, ws)
        M.mgrit_pack(self.keep, self.Y, self.Y8)
        M.mgrit_cross_entropy(self.loss, self.logits, self.labels, self.value, None, self.logits, ws)
        M.mgrit_affine_kept_backward(self.head, self.Y8, p["Wo"], None, self.logits, self.Y, g["Wo"], g["bo"], ws)       # (Y's gradient in its place)
        M.mgrit_block_norm_backward(self.norm, self.f, self.S, p["gate"], p["post"], p["pre"], None, self.Y, self.df, self.dr, g["gate"], g["post"],
                                    g["pre"], ws)
        M.mgrit_affine_kept_backward(self.block, self.u8, p["Wb"], self.D8, self.df, self.lamN, g["Wb"], g["bb"], ws)
        self.lamN.add_(self.dr)
        M.mgrit_fas_adjoint(self.stack, p["W"], p["b"], self.U, self.lamN, self.Lam, g["W"], g["b"], ws, want_hist=False)

    def exact(self):
        """The same in 64 bits: autograd, but that the products of the backward pass take the activations that came back from 8 bits."""
        class Kept(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x, W, b, x8, D8, act):
                ctx.save_for_backward(W, x8, D8)
                z = x @ W.T + b
                return torch.tanh(z) if act else z

            @staticmethod
            def backward(ctx, dy):
                W, x8, D8 = ctx.saved_tensors
                G = dy * D8
                return G @ W, G.T @ x8, G.sum(0), None, None, None

        p = {k: v.double().requires_grad_() for k, v in self.par.items()}
        come_back = lambda a: unpacked(self.keep, a, "f").double()                                     # noqa: E731
        u = self.u0.double()
        for n in range(self.N):
            u = u + torch.tanh(u @ p["W"][n].T + p["b"][n]) / self.N
        f = Kept.apply(u, p["Wb"], p["bb"], come_back(self.u8), come_back(self.D8), True)
        S = u + STEP * p["gate"] * norm_of(f, "rms", EPS)[0] * p["post"]
        Y = norm_of(S, "rms", EPS)[0] * p["pre"]
        z = Kept.apply(Y, p["Wo"], p["bo"], come_back(self.Y8), torch.ones((), device="cuda", dtype=torch.float64), False)
        loss = (torch.logsumexp(z, 1) - z.gather(1, self.labels[:, None])[:, 0]).mean()
        loss.backward()
        return float(loss.detach()), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("B,q,N,classes", [(24, 64, 8, 10), (40, 136, 5, 33)])
def test_a_training_step_with_kept_activations(B, q, N, classes):
    net = Network(B, q, N, classes)
    net.step()
    loss, grad = net.exact()
    # a chain of N + 4 products and norms of at most q terms and their transposes: relative errors of (a few) sqrt(terms) 2^-24 each
    tol = 2 * (N + 4) * (4 * q) ** 0.5 * 2.0 ** -24
    assert abs(float(net.value) - loss) <= tol * abs(loss)
    for k, g in grad.items():
        err = float((net.grad[k].double() - g).norm() / g.norm())
        assert err <= tol, (k, err, tol)


def test_a_captured_step_replays_beside_eager_work():
    net = Network(16, 72, 4, 10)
    net.step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        net.step()
    for replay in range(3):
        for k, v in net.par.items():
            v.add_(normal(v.shape, 0.01, "f", 30 + replay))
        net.step()
        want = [net.value.clone()] + [g.clone() for g in net.grad.values()]
        for g in net.grad.values():
            g.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip([net.value] + list(net.grad.values()), want)), replay


@pytest.mark.parametrize("B", [1, 17, 200])
@pytest.mark.parametrize("form", ["bf16", "mx4"])
def test_answers_from_packed_weights(B, form):
    """Norm, a head of many classes with weights in 4 bits, one class a row."""
    q, V = 320, 5003
    f, r, pre = normal((B, q), 1.0, "b", 1), normal((B, q), 1.0, "f", 2), 1.0 + normal((q,), 0.1, "f", 3)
    W, w4 = packed(normal((V, q), 2.0 * q ** -0.5, "b", 4), "mx4")
    n = M.make_block_norm(M=B, q=q, ftype=M.MGRIT_BF16, eps=EPS, scale=STEP)
    p = M.make_affine_packed(M=B, K=q, F=V, xtype=M.MGRIT_BF16, xformat=M.MGRIT_MX4 if form == "mx4" else M.MGRIT_BF16)
    s = M.make_sample(B=B, V=V)
    S, Y, logits = torch.empty_like(r), torch.empty_like(f), torch.empty((B, V), device="cuda")
    index, logprob = torch.empty((B,), dtype=torch.int64, device="cuda"), torch.empty((B,), device="cuda")
    ws = torch.empty(M.mgrit_affine_packed_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    u, t, k, top = uniform(B, 5), uniform(B, 6, 0.5, 1.5), whole(B, 1, 200, 7), uniform(B, 8, 0.5, 1.0)
    M.mgrit_block_norm_forward(n, f, r, None, None, pre, S, Y)
    M.mgrit_affine_packed_forward(p, Y, w4, None, None, logits, None, ws)
    M.mgrit_sample(s, logits, u, t, k, top, None, index, logprob, None)
    want = norm_of(r.double() + STEP * f.double(), "rms", EPS)[0] * pre.double()
    near(Y, want, 2.0 ** -20 * want.abs(), "Y")
    if form == "mx4":
        y, y4 = packed(Y, "mx4")
        Yv = unpacked(y, y4, "f").double()
    else:
        Yv = Y.double()
    Wv = unpacked(W, w4, "f").double()
    near(logits, Yv @ Wv.T, (q + 8) * 2.0 ** -23 * (Yv.abs() @ Wv.abs().T), "logits")
    for b in range(0, B, max(1, B // 8)):
        v, lp, border = answer(logits[b].cpu(), float(u[b]), float(t[b]), int(k[b]), float(top[b]), 0.0)
        assert int(index[b]) == v or border < 1.0e-12
        assert abs(float(logprob[b]) - lp) <= 2.0 ** -24 * abs(lp) + 1.0e-11 or int(index[b]) != v

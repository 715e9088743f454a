"""The operators around the solver as they are used: opening layer, stack, closing layer, loss, and all of it backwards, clipped to a
norm.  Every gradient against autograd in 64 bits through the same network, serially."""
import math

import pytest
import torch

import paper_2007_07336_amd as M
from tests.ops_util import normal

pytestmark = pytest.mark.gpu


class Network:
    """28 x 28 images (or any `pixels`) -> q features -> N residual layers -> classes"""

    def __init__(self, B, pixels, q, N, classes, act, act_open):
        self.B, self.q, self.N, self.act_open, self.act = B, q, N, act_open, act
        f = lambda *s: torch.zeros(s, device="cuda")                                                # noqa: E731
        self.x, self.labels = normal((B, pixels), 1.0, "f", 1), torch.randint(0, classes, (B,), generator=torch.Generator().manual_seed(2)).cuda()
        self.labels[::5] = -1
        self.par = {"Wi": normal((q, pixels), pixels ** -0.5, "f", 3), "bi": normal((q,), 0.3, "f", 4), "W": normal((N, q, q), q ** -0.5, "f", 5),
                    "b": normal((N, q), 0.3, "f", 6), "Wo": normal((classes, q), q ** -0.5, "f", 7), "bo": normal((classes,), 0.3, "f", 8)}
        self.grad = {k: torch.full_like(v, float("nan")) for k, v in self.par.items()}
        # levels = 1: serial propagation, so that the solves are exact and the whole step can be compared to rounding
        self.stack = M.make_problem(N=N, h=1.0 / N, m=4, max_levels=1, relax=0, max_iter=1, layer=0, act=act, dtype=0, B=B, q=q)
        self.open = M.make_affine(M=B, K=pixels, F=q, act=act_open)
        self.close = M.make_affine(M=B, K=q, F=classes)
        self.loss = M.make_loss(B=B, V=classes)
        self.U, self.Lam, self.D, self.logits = f(N + 1, B, q), f(N + 1, B, q), f(B, q), f(B, classes)
        self.lamN, self.u0, self.value = f(B, q), f(B, q), f(1)
        self.tensors = M.make_tensor_list(list(self.grad.values()))
        self.norm = f(1)
        n = max(M.mgrit_adjoint_workspace_bytes(self.stack), M.mgrit_affine_workspace_bytes(self.open), M.mgrit_affine_workspace_bytes(self.close),
                M.mgrit_affine_backward_workspace_bytes(self.open), M.mgrit_affine_backward_workspace_bytes(self.close),
                M.mgrit_cross_entropy_workspace_bytes(self.loss), M.mgrit_clip_workspace_bytes(self.tensors))
        self.ws = torch.empty(n, dtype=torch.uint8, device="cuda")           # one workspace: the calls follow one another on one stream

    def step(self, max_norm):
        p, g = self.par, self.grad
        M.mgrit_affine_forward(self.open, self.x, p["Wi"], p["bi"], None, self.u0, self.D, self.ws)
        M.mgrit_fas_forward(self.stack, p["W"], p["b"], self.u0, self.U, self.ws, want_hist=False)
        M.mgrit_affine_forward(self.close, self.U[self.N], p["Wo"], p["bo"], None, self.logits, None, self.ws)
        M.mgrit_cross_entropy(self.loss, self.logits, self.labels, self.value, None, self.logits, self.ws)
        M.mgrit_affine_backward(self.close, self.U[self.N], p["Wo"], None, self.logits, self.lamN, g["Wo"], g["bo"], self.ws)
        M.mgrit_fas_adjoint(self.stack, p["W"], p["b"], self.U, self.lamN, self.Lam, g["W"], g["b"], self.ws, want_hist=False)
        M.mgrit_affine_backward(self.open, self.x, None, self.D if self.act_open != M.MGRIT_ACT_IDENTITY else None, self.Lam[0], None, g["Wi"], g["bi"],
                                self.ws)
        M.mgrit_clip_gradients(self.tensors, max_norm, self.norm, self.ws)

    def exact(self):
        act = {M.MGRIT_ACT_TANH: torch.tanh, M.MGRIT_ACT_RELU: torch.relu, M.MGRIT_ACT_IDENTITY: lambda z: z}
        p = {k: v.double().requires_grad_() for k, v in self.par.items()}
        u = act[self.act_open](self.x.double() @ p["Wi"].T + p["bi"])
        for n in range(self.N):
            u = u + act[self.act](u @ p["W"][n].T + p["b"][n]) / self.N
        rows = torch.logsumexp(u @ p["Wo"].T + p["bo"], 1) - (u @ p["Wo"].T + p["bo"]).gather(1, self.labels.clamp(min=0)[:, None])[:, 0]
        loss = rows[self.labels >= 0].mean()
        loss.backward()
        return float(loss.detach()), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("B,pixels,q,N,act_open", [(32, 784, 64, 16, M.MGRIT_ACT_TANH), (7, 50, 24, 9, M.MGRIT_ACT_IDENTITY)])
def test_a_training_step(B, pixels, q, N, act_open):
    net = Network(B, pixels, q, N, 10, M.MGRIT_ACT_TANH, act_open)
    loss, grad = net.exact()
    norm = math.sqrt(sum(float((g ** 2).sum()) for g in grad.values()))
    net.step(norm / 3)
    # a chain of N + 2 products of at most 784 terms and their transposes: relative errors of (a few) sqrt(terms) 2^-24 each
    tol = 2 * (N + 2) * math.sqrt(784) * 2.0 ** -24
    assert abs(float(net.value) - loss) <= tol * abs(loss)
    assert abs(float(net.norm) - norm) <= tol * norm
    for k, g in grad.items():
        err = float((net.grad[k].double() * 3 - g).norm() / g.norm())
        assert err <= tol, (k, err)


def test_a_captured_training_step_replays_beside_eager_work():
    net = Network(16, 100, 32, 8, 10, M.MGRIT_ACT_RELU, M.MGRIT_ACT_RELU)
    net.step(0.5)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        net.step(0.5)
    for replay in range(3):
        for k, v in net.par.items():
            v.add_(normal(v.shape, 0.01, "f", 30 + replay))                  # an update in place, seen by the graph
        net.step(0.5)
        want = [net.value.clone(), net.norm.clone()] + [g.clone() for g in net.grad.values()]
        for g in net.grad.values():
            g.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip([net.value, net.norm] + list(net.grad.values()), want):
            assert torch.equal(t, w), replay
